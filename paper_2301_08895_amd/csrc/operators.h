// Shared by the operators of a network's hidden layers (kernels_linear.hip, kernels_norm.hip, kernels_dropout.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "abs_common.h"

namespace abs_impl {

// Sets the text abs_last_error(NULL) returns on this thread; returns `code`.
int op_fail(int code, const char* text) noexcept;
int op_hip(const char* what, hipError_t e) noexcept;     // ABS_OK for hipSuccess

inline size_t op_round_up(size_t x, size_t m) { return (x + m - 1) / m * m; }
inline bool op_aligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
inline int op_size(int dtype) { return dtype == ABS_X_BF16 ? 2 : 4; }

// A grid of `blocks` workgroups for kernels that go by op_block(): a dimension of a launch counts its work-items in 32 bits,
// so many workgroups are laid out over two.  The last row may hold workgroups beyond the count: the kernels check.
inline dim3 op_grid(uint64_t blocks) {
  constexpr uint64_t row = 1u << 20;
  return blocks <= row ? dim3((unsigned)blocks) : dim3((unsigned)row, (unsigned)((blocks + row - 1) / row));
}

#if defined(__HIPCC__)
__device__ __forceinline__ uint64_t op_block() { return (uint64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// ---- elements: bf16 travels as its 16 bits -----------------------------------------------------------
__device__ __forceinline__ float op_widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float op_widen(float v) { return v; }
// round to nearest even; gfx950 has the instruction, a NaN stays one
__device__ __forceinline__ uint16_t op_bf16(float f) {
  const __bf16 h = (__bf16)f;
  uint16_t r;
  __builtin_memcpy(&r, &h, 2);
  return r;
}
__device__ __forceinline__ void op_narrow(float f, uint16_t& v) { v = op_bf16(f); }
__device__ __forceinline__ void op_narrow(float f, float& v) { v = f; }

// V elements that are loaded and stored as one piece
template <typename T, int V>
struct alignas(sizeof(T) * V) OpVec { T e[V]; };

// ---- activations.  act(z) and act'(z) in fp32; a NaN stays one ----------------------------------------
__device__ __forceinline__ float op_sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }   // 2 ulp
template <int ACT>
__device__ __forceinline__ float op_act(float z) {
  if (ACT == ABS_ACT_RELU) return z < 0.f ? 0.f : z;
  if (ACT == ABS_ACT_SILU) return z * op_sigmoid(z);
  if (ACT == ABS_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
  return z;
}
template <int ACT>
__device__ __forceinline__ float op_act_slope(float z) {
  if (ACT == ABS_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (ACT == ABS_ACT_SILU) { const float p = op_sigmoid(z); return p * (1.0f + z * (1.0f - p)); }
  if (ACT == ABS_ACT_GELU)
    return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * __expf(-0.5f * z * z) * 0.39894228040143268f;
  return 1.f;
}
// the same with the activation as a uniform run-time value
__device__ __forceinline__ float op_act(float z, int act) {
  switch (act) {
    case ABS_ACT_RELU: return op_act<ABS_ACT_RELU>(z);
    case ABS_ACT_SILU: return op_act<ABS_ACT_SILU>(z);
    case ABS_ACT_GELU: return op_act<ABS_ACT_GELU>(z);
    default: return z;
  }
}
__device__ __forceinline__ float op_act_slope(float z, int act) {
  switch (act) {
    case ABS_ACT_RELU: return op_act_slope<ABS_ACT_RELU>(z);
    case ABS_ACT_SILU: return op_act_slope<ABS_ACT_SILU>(z);
    case ABS_ACT_GELU: return op_act_slope<ABS_ACT_GELU>(z);
    default: return 1.f;
  }
}
#endif

}  // namespace abs_impl
