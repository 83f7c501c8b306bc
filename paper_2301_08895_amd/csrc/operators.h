// Shared by the operators of a network's hidden layers (kernels_linear.hip, kernels_norm.hip, kernels_dropout.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "abs_common.h"

namespace abs_impl {

// Sets the text abs_last_error(NULL) returns on this thread; returns `code`.
int op_fail(int code, const char* text) noexcept;
int op_hip(const char* what, hipError_t e) noexcept;     // ABS_OK for hipSuccess

// A product left as the fp32 shares of its contraction: element (m, n) is the sum over k < shares of part[k stride + m ld + n], in that order.
struct OpShares { const float* part; int64_t ld, stride; int shares; };
// abs_linear_forward's x W and abs_linear_backward with dW left so (in d_workspace, until something else is done there), for sums that are used in
// fp32 at once; d_dx and d_db may be NULL.  op_linear_shares_size(): what they need of d_workspace, at any alignment of the operands.
size_t op_linear_shares_size(const abs_linear* p, int32_t backward) noexcept;
int op_linear_forward_shares(const abs_linear* p, const void* d_x, const void* d_w, void* d_workspace, size_t workspace_bytes, void* hip_stream,
                             OpShares* product) noexcept;
int op_linear_backward_shares(const abs_linear* p, const void* d_x, const void* d_w, const void* d_z, const void* d_dy, void* d_dx, float* d_db,
                              void* d_workspace, size_t workspace_bytes, void* hip_stream, OpShares* dw) noexcept;

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

// N consecutive elements at any alignment of theirs, loaded or stored as one access (the memory system takes it at any address)
template <typename T, int N> struct __attribute__((packed, aligned(sizeof(T)))) Loose { T e[N]; };

// V elements held in whole registers: left as an array of 16-bit elements the compiler gives every one a register of its own.
template <typename T, int V>
struct Piece {
  static constexpr int kBytes = V * (int)sizeof(T), kWords = kBytes < 4 ? 1 : kBytes / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const void* p) {
    if constexpr (kBytes < 4) w[0] = *(const uint16_t*)p;
    else { const Loose<T, V> l = *(const Loose<T, V>*)p; __builtin_memcpy(w, &l, kBytes); }
  }
  __device__ __forceinline__ float at(int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else return __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
  }
  // forgets what has been computed from the words: they are widened again, not kept widened
  __device__ __forceinline__ void hide() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) asm volatile("" : "+v"(w[i]));
  }
  __device__ __forceinline__ void set(const float* f) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] = __float_as_uint(f[e]);
    } else if constexpr (V == 1) {
      w[0] = op_bf16(f[0]);
    } else {
      typedef float f32x2 __attribute__((ext_vector_type(2)));
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        const bf16x2 h = __builtin_convertvector(f32x2{f[2 * i], f[2 * i + 1]}, bf16x2);
        __builtin_memcpy(&w[i], &h, 4);
      }
    }
  }
  __device__ __forceinline__ void store(void* p) const {
    if constexpr (kBytes < 4) *(uint16_t*)p = (uint16_t)w[0];
    else { Loose<T, V> l; __builtin_memcpy(&l, w, kBytes); *(Loose<T, V>*)p = l; }
  }
};

// ---- activations.  act(z) and act'(z) in fp32; a NaN stays one.  u = 2^-24 is half a step of fp32 ---------------
// Two evaluations of each: behind fp32 elements (kFine) one that is off by a few steps of the result at every z, behind bf16 ones, whose
// half step is 2^-8, one of half as many operations.
template <typename T> constexpr bool kFine = sizeof(T) == 4;

// exp(-s) (1 - c), s in [0, 400], c small: the product s log2(e) in two parts, so that its rounding does not grow with s.
__device__ __forceinline__ float op_exp_minus(float s, float c) {
  constexpr float kLog2e = 1.44269502f, kRest = 1.92596303e-8f, kLn2 = 0.693147182f;
  const float y = s * kLog2e, low = fmaf(s, kRest, fmaf(s, kLog2e, -y));
  const float e = __builtin_amdgcn_exp2f(-y);
  return fmaf(-fmaf(low, kLn2, c), e, e);
}
// The logistic function p = 1 / (1 + exp(-z)) and q = 1 - p.  Fine: 6 u of either at every z.  Else p's error is a few u of p for z >= 0 and
// grows to about |z| u of p below (the rounding of z log2(e)): a few u of 1, and 2^-18 of p where z = -80.
template <bool FINE>
__device__ __forceinline__ float op_sigmoid(float z, float& q) {
  if (FINE) {
    const float e = op_exp_minus(fminf(fabsf(z), 200.f), 0.f), r = __builtin_amdgcn_rcpf(1.0f + e), er = e * r;
    q = z < 0.f ? r : er;
    return z < 0.f ? er : r;
  }
  const float p = __builtin_amdgcn_rcpf(1.0f + __expf(-z));
  q = 1.0f - p;
  return p;
}
// The normal distribution function Phi(z) = (1 + erf(z / sqrt 2)) / 2, and e = exp(-z^2 / 2), which the slope's density needs too.
// Fine: Phi(-x) = e f(x), x = |z|, where f(x) (x + 5/2) is smooth and between 1/2 and 5/4: a polynomial of degree 9 in (x - 5/2) / (x + 5/2) (fitted to
// [0, 13.6] for the least largest relative error, 0.25 u), e with x^2 in two parts.  10 u of Phi at every z, in 34 operations.
// Else erfc by the rational form in t = 1 / (1 + p |z| / sqrt 2) of Abramowitz and Stegun, 7.1.26: erf's error is 1.5e-7 at most (a
// relative error of Phi of 2^-14 at z = -3), in 13 operations; two more in either are transcendental.
template <bool FINE>
__device__ __forceinline__ float op_phi(float z, float& e) {
  float tail;                                            // Phi(-|z|)
  if (FINE) {
    const float x = fminf(fabsf(z), 20.f), h = 0.5f * x, s = h * x;
    e = op_exp_minus(s, fmaf(h, x, -s));
    const float t = __builtin_amdgcn_rcpf(x + 2.5f), v = fmaf(-5.0f, t, 1.0f);
    float f = -0.000156221766f;
    f = fmaf(f, v, -0.000309014693f);
    f = fmaf(f, v, 0.000684247119f);
    f = fmaf(f, v, 0.00252179429f);
    f = fmaf(f, v, -0.00160130544f);
    f = fmaf(f, v, -0.0163856447f);
    f = fmaf(f, v, 0.00923601165f);
    f = fmaf(f, v, 0.131986931f);
    f = fmaf(f, v, -0.433692008f);
    f = fmaf(f, v, 0.706656635f);
    tail = f * t * e;
  } else {
    const float x = fabsf(z) * 0.70710678118654752f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.0f));
    e = __expf(-x * x);
    const float q = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    tail = 0.5f * q * e;
  }
  return z < 0.f ? tail : 1.0f - tail;
}
template <int ACT, bool FINE>
__device__ __forceinline__ float op_act(float z) {
  if (ACT == ABS_ACT_RELU) return z < 0.f ? 0.f : z;
  if (ACT == ABS_ACT_SILU) { float q; return z * op_sigmoid<FINE>(z, q); }
  if (ACT == ABS_ACT_GELU) { float e; return z * op_phi<FINE>(z, e); }
  return z;
}
// d act'(z).  relu: a choice, not a product - nothing of d passes where z is not positive, and it may be infinite there
template <int ACT, bool FINE>
__device__ __forceinline__ float op_slope(float d, float z) {
  if (ACT == ABS_ACT_RELU) return z > 0.f ? d : 0.f;
  if (ACT == ABS_ACT_SILU) { float q; const float p = op_sigmoid<FINE>(z, q); return d * fmaf(z * p, q, p); }
  if (ACT == ABS_ACT_GELU) { float e; const float c = op_phi<FINE>(z, e); return d * fmaf(z * 0.39894228040143268f, e, c); }
  return d;
}
// N values at once, the activation a uniform run-time value: one branch
template <int N, bool FINE>
__device__ __forceinline__ void op_act_all(float* h, int act) {
  asm volatile("" : "+s"(act));           // (compared here: not once, with the result kept in scalar registers)
  if (act == ABS_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) h[i] = op_act<ABS_ACT_RELU, FINE>(h[i]);
  } else if (act == ABS_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) h[i] = op_act<ABS_ACT_SILU, FINE>(h[i]);
  } else if (act == ABS_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) h[i] = op_act<ABS_ACT_GELU, FINE>(h[i]);
  }
}
// d[i] = d[i] act'(h[i])
template <int N, bool FINE>
__device__ __forceinline__ void op_slope_all(float* d, const float* h, int act) {
  asm volatile("" : "+s"(act));
  if (act == ABS_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = op_slope<ABS_ACT_RELU, FINE>(d[i], h[i]);
  } else if (act == ABS_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = op_slope<ABS_ACT_SILU, FINE>(d[i], h[i]);
  } else if (act == ABS_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = op_slope<ABS_ACT_GELU, FINE>(d[i], h[i]);
  }
}
// the same with the activation as a uniform run-time value
template <bool FINE>
__device__ __forceinline__ float op_act(float z, int act) {
  switch (act) {
    case ABS_ACT_RELU: return op_act<ABS_ACT_RELU, FINE>(z);
    case ABS_ACT_SILU: return op_act<ABS_ACT_SILU, FINE>(z);
    case ABS_ACT_GELU: return op_act<ABS_ACT_GELU, FINE>(z);
    default: return z;
  }
}
template <bool FINE>
__device__ __forceinline__ float op_slope(float d, float z, int act) {
  switch (act) {
    case ABS_ACT_RELU: return op_slope<ABS_ACT_RELU, FINE>(d, z);
    case ABS_ACT_SILU: return op_slope<ABS_ACT_SILU, FINE>(d, z);
    case ABS_ACT_GELU: return op_slope<ABS_ACT_GELU, FINE>(d, z);
    default: return d;
  }
}
#endif

}  // namespace abs_impl
