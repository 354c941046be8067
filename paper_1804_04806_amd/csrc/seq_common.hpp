// What the sequence operators' kernels share: element types, wide loads, activations, sums over lanes.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace ucd {
namespace seq {

typedef __bf16 bf16_t;

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16_t v) { return (float)v; }
template <class T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t from_f<bf16_t>(float v) { return (bf16_t)v; }   // to nearest, ties to even

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// 1 / (1 + exp(-v)).  exp(-v) overflows to infinity below -88: the quotient is then 0, as it should be.
__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + __expf(-v)); }

}  // namespace seq
}  // namespace ucd
