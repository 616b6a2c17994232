// Microscaled 4-bit floats (MXFP4: E2M1 values, an E8M0 scale per 32): what the kernels that make and use them share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>
#include <stdint.h>

#include "common.cuh"

namespace slicemoe {

constexpr int kMxBlock = 32;    // values that share a scale
constexpr int kMxRows = 128;    // rows of a block of the packed layout
constexpr int kMxChunk = 64;    // values of a chunk: what one tensor instruction contracts
constexpr int kMxChunkBytes = kMxRows * kMxChunk / 2;
constexpr int kMxAtomK = 128;   // values whose scales lie together
constexpr int kMxAtomBytes = kMxRows * kMxAtomK / kMxBlock;
constexpr int kMxMaxN = 1 << 21, kMxMaxK = 1 << 20;
constexpr int kMxMaxRow = 1 << 30;  // values of a row, and rows, of the calls without matrices: counters that step past them stay within an int

__host__ __device__ inline int mx_chunks(int K) { return (K + kMxChunk - 1) / kMxChunk; }
__host__ __device__ inline int mx_atoms(int K) { return (K + kMxAtomK - 1) / kMxAtomK; }
__host__ __device__ inline int mx_pitch(int K) { return 4 * mx_atoms(K); }
// Rows of the packed layout: of a gated pair 16 of gate and 16 of up in turn.
__host__ __device__ inline int mx_phys_rows(int N, int gated) { return gated ? 32 * ((N + 15) / 16) : N; }
__host__ __device__ inline int mx_row_blocks(int N, int gated) { return (mx_phys_rows(N, gated) + kMxRows - 1) / kMxRows; }
// Where block kb (32 values, 16 bytes of codes) of a physical row lies, and its scale byte.
__host__ __device__ inline size_t mx_code_offset(int K, int row, int kb) {
  return ((size_t)(row / kMxRows) * mx_chunks(K) + (kb >> 1)) * kMxChunkBytes + (size_t)(kb & 1) * (kMxRows * 16) + (size_t)(row % kMxRows) * 16;
}
__host__ __device__ inline size_t mx_scale_offset(int K, int row, int kb) {
  const int r = row % kMxRows;
  return ((size_t)(row / kMxRows) * mx_atoms(K) + (kb >> 2)) * kMxAtomBytes + (size_t)(r & 31) * 16 + (size_t)(r >> 5) * 4 + (kb & 3);
}

inline bool mx_dtype(int d) { return d == SLICEMOE_F32 || d == SLICEMOE_BF16 || d == SLICEMOE_F16; }
inline size_t mx_elem(int d) { return d == SLICEMOE_F32 ? 4 : 2; }
inline bool mx_aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// The scale byte of a block from the bits of its largest magnitude (as fp32): the exponent less 2, the exponent of the largest
// 4-bit value.  An infinity or NaN among the values makes it 255.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_bits) {
  const uint32_t ex = amax_bits >> 23;
  return ex == 255u ? 255u : (ex > 2u ? ex - 2u : 0u);
}
// The factor that undoes a scale, 2^(127 - b); a NaN block's codes are 0.
__device__ __forceinline__ float mx_inverse(uint32_t b) { return b == 255u ? 0.0f : __uint_as_float((254u - b) << 23); }
__device__ __forceinline__ float mx_scale_value(uint32_t b) {
  return b == 0u ? __uint_as_float(0x00400000u) : (b == 255u ? CUDART_NAN_F : __uint_as_float(b << 23));
}
// Eight values, scaled exactly (a power of two), to eight 4-bit floats: round to nearest even, saturating.
__device__ __forceinline__ uint32_t mx_encode8(const float (&v)[8], float inv) {
  uint32_t r;
  asm("{\n .reg .b8 a, b, c, d;\n"
      " cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
      " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
      " mov.b32 %0, {a, b, c, d};\n}"
      : "=r"(r)
      : "f"(v[0] * inv), "f"(v[1] * inv), "f"(v[2] * inv), "f"(v[3] * inv), "f"(v[4] * inv), "f"(v[5] * inv), "f"(v[6] * inv),
        "f"(v[7] * inv));
  return r;
}
// Two 4-bit floats (the low byte of a word's) as two fp16.
__device__ __forceinline__ __half2 mx_decode2(uint32_t byte) {
  uint32_t r;
  asm("{\n .reg .b8 a, z1, z2, z3;\n mov.b32 {a, z1, z2, z3}, %1;\n cvt.rn.f16x2.e2m1x2 %0, a;\n}" : "=r"(r) : "r"(byte));
  return *reinterpret_cast<__half2*>(&r);
}

template <class T>
__device__ __forceinline__ float mx_to_float(T v);
template <>
__device__ __forceinline__ float mx_to_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ float mx_to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float mx_to_float<__half>(__half v) { return __half2float(v); }
template <class T>
__device__ __forceinline__ T mx_from_float(float v);
template <>
__device__ __forceinline__ float mx_from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 mx_from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half mx_from_float<__half>(float v) { return __float2half_rn(v); }

// One element, read past L1: a kernel that is launched early may run on an SM whose L1 still holds what the address held before.
__device__ __forceinline__ float mx_load(const float* p) { return __ldcg(p); }
__device__ __forceinline__ float mx_load(const __nv_bfloat16* p) {
  return __uint_as_float((uint32_t)__ldcg(reinterpret_cast<const unsigned short*>(p)) << 16);
}
__device__ __forceinline__ float mx_load(const __half* p) { return __half2float(__ushort_as_half(__ldcg(reinterpret_cast<const unsigned short*>(p)))); }

// Eight consecutive elements as floats (past L1 too), and back; WIDE: by 16-byte accesses (the address is a multiple of 16), else one by one.
template <class T, bool WIDE>
__device__ __forceinline__ void mx_load8(const T* p, float (&v)[8]) {
  if constexpr (!WIDE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = mx_load(p + i);
  } else if constexpr (sizeof(T) == 4) {
    const float4 a = __ldcg(reinterpret_cast<const float4*>(p)), b = __ldcg(reinterpret_cast<const float4*>(p) + 1);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else {
    const uint4 a = __ldcg(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      T e[2];
      memcpy(e, &w[i], 4);
      v[2 * i] = mx_to_float<T>(e[0]), v[2 * i + 1] = mx_to_float<T>(e[1]);
    }
  }
}
template <class T, bool WIDE>
__device__ __forceinline__ void mx_store8(T* p, const float (&v)[8]) {
  if constexpr (!WIDE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = mx_from_float<T>(v[i]);
  } else if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const T e[2] = {mx_from_float<T>(v[2 * i]), mx_from_float<T>(v[2 * i + 1])};
      memcpy(&w[i], e, 4);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// A launch that may start while the kernel before it on the stream is still running; the kernel waits for it itself.
template <class... Args>
static int mx_launch(void (*kernel)(Args...), dim3 blocks, unsigned threads, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = blocks;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  SM_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, args...));
  return SLICEMOE_OK;
}
__device__ __forceinline__ void mx_dep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void mx_dep_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

}  // namespace slicemoe
