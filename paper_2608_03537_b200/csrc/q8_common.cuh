// What the kernels of the 8-bit integer layers share: element types, wide accesses, activations.
#pragma once

#include <cuda_fp16.h>

#include "comfuse.h"
#include "sm100_primitives.cuh"

namespace comfuse {

// An element type (comfuse_dtype_t) in memory; everything is computed in fp32.
template <int DT>
struct Elem {
  static constexpr int kBytes = DT == COMFUSE_DTYPE_F32 ? 4 : 2;
  using Word = typename std::conditional<DT == COMFUSE_DTYPE_F32, uint32_t, uint16_t>::type;
  static __device__ __forceinline__ float get(const void* p, long long i) {
    const Word w = static_cast<const Word*>(p)[i];
    if constexpr (DT == COMFUSE_DTYPE_F32) return __uint_as_float(w);
    else if constexpr (DT == COMFUSE_DTYPE_BF16) return __uint_as_float(static_cast<uint32_t>(w) << 16);
    else return __half2float(__ushort_as_half(w));
  }
  static __device__ __forceinline__ void put(void* p, long long i, float v) {
    if constexpr (DT == COMFUSE_DTYPE_F32) static_cast<Word*>(p)[i] = __float_as_uint(v);
    else if constexpr (DT == COMFUSE_DTYPE_BF16) static_cast<Word*>(p)[i] = static_cast<Word>(pack_bf16x2_rn(v, 0.f));
    else static_cast<Word*>(p)[i] = static_cast<Word>(pack_f16x2_rn(v, 0.f));
  }
  // element i of packed words
  static __device__ __forceinline__ float of(const uint32_t* w, int i) {
    if constexpr (DT == COMFUSE_DTYPE_F32) return __uint_as_float(w[i]);
    else if constexpr (DT == COMFUSE_DTYPE_BF16) return (i & 1) ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
    else return __half2float(__ushort_as_half(static_cast<uint16_t>((i & 1) ? w[i >> 1] >> 16 : w[i >> 1] & 0xFFFFu)));
  }
  // N elements into packed words
  template <int N>
  static __device__ __forceinline__ void pack(const float (&v)[N], uint32_t* w) {
    if constexpr (DT == COMFUSE_DTYPE_F32) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = __float_as_uint(v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) w[i] = DT == COMFUSE_DTYPE_BF16 ? pack_bf16x2_rn(v[2 * i], v[2 * i + 1]) : pack_f16x2_rn(v[2 * i], v[2 * i + 1]);
    }
  }
};

// No load of these kernels takes the read-only path (__ldg): with programmatic launch they are on the SMs while the kernels in front of them
// still write scales and rows, and that path is for data that nobody writes while a kernel runs; it may also be an output, in place.
// Data that is read or written once, by one thread: past the L1.
__device__ __forceinline__ void ld_16(const void* p, uint32_t* w) {
  asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p) : "memory");
}
__device__ __forceinline__ void st_16(void* p, const uint32_t* w) {
  asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}
__device__ __forceinline__ void ld_8(const void* p, uint32_t* w) {
  asm volatile("ld.global.L1::no_allocate.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p) : "memory");
}
__device__ __forceinline__ void st_8(void* p, const uint32_t* w) {
  asm volatile("st.global.v2.b32 [%0], {%1, %2};" ::"l"(p), "r"(w[0]), "r"(w[1]) : "memory");
}
// 1 / (1 + e^-x) from ex2 and rcp.  Relative error: ex2 2^-22, the addition 2^-24, rcp 2^-23, and |x| 2^-23 of the exponent (its product's rounding
// and that of log2 e): below 2^-21 + |x| 2^-23.  A result below 2^-126 (x < -87.3) is 0: rcp flushes it.
__device__ __forceinline__ float sigmoid_f32(float x) { return rcp_approx(1.f + ex2_approx(x * -1.4426950408889634f)); }

// The activations of the library's reduction-free kinds on N values.  GELU's 0.5 (1 + tanh u) is the sigmoid of 2u: two special-function
// instructions, but relatively exact in the left tail, where 1 + tanh.approx cancels (z = -3: 20 % off), and Y may be fp32.
template <int N>
__device__ __forceinline__ void activate(float (&z)[N], int activation) {
  switch (activation) {
    case COMFUSE_OP_RELU:
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = z[i] < 0.f ? 0.f : z[i];  // (a NaN stays one)
      break;
    case COMFUSE_OP_GELU_TANH:
#pragma unroll
      for (int i = 0; i < N; ++i) {
        constexpr float c = 2.f * 0.7978845608028654f;
        z[i] *= sigmoid_f32(z[i] * fmaf(c * 0.044715f, z[i] * z[i], c));
      }
      break;
    case COMFUSE_OP_TANH:
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = tanhf(z[i]);
      break;
    case COMFUSE_OP_SIGMOID:
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = sigmoid_f32(z[i]);
      break;
    default: break;
  }
}

}  // namespace comfuse
