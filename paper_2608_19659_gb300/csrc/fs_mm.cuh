// Shared parts of the products of a rank's layer (fs_mm.cu and its kernels).
#pragma once

#include "fs_kv.cuh"

namespace fs {

// What a product's epilogue reads and writes. Rows are the call's rows (tokens), columns what W's rows are.
struct MmEpilogue {
  int rows, cols, act;
  const float* x_scale;     // e4m3: of each row, else null
  const float* w_scale[2];  // of each column (of gate and up)
  const void* bias;
  const void* in;  // residual, or dy of the backward pass
  long long in_stride;
  void* out[2];  // y; dg and du in the backward pass
  long long out_stride;
};

// z / (1 + e^-2h), 2 log2(e) h in `e`: the logistic function's share of z. The quotient is
// off by 2 ulp, and 0 where e^-2h passes 2^126 (values under 2^-119 of z).
__device__ __forceinline__ float mm_logistic(float z, float e) { return __fdividef(z, 1.f + ex2(-e)); }

constexpr float kLog2e = 1.44269504f, kTanhC = 0.7978845608f, kTanhD = 0.044715f;

// Phi(z) by the complementary error function: no cancellation in the lower tail.
__device__ __forceinline__ float mm_phi(float z) { return 0.5f * erfcf(-0.70710678f * z); }

template <int kAct>
__device__ __forceinline__ float mm_act(float z) {
  if (kAct == FS_ACT_RELU) return z < 0.f ? 0.f : z;  // (a NaN stays one)
  if (kAct == FS_ACT_SILU) return mm_logistic(z, kLog2e * z);
  if (kAct == FS_ACT_GELU) return z * mm_phi(z);
  // (1 + tanh h) / 2 is the logistic function of 2 h
  if (kAct == FS_ACT_GELU_TANH) return mm_logistic(z, 2.f * kLog2e * kTanhC * (z + kTanhD * z * z * z));
  return z;
}

// act(z), and its slope there.
template <int kAct>
__device__ __forceinline__ float mm_act_slope(float z, float& slope) {
  if (kAct == FS_ACT_RELU) {
    slope = z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
    return z < 0.f ? 0.f : z;
  }
  if (kAct == FS_ACT_SILU) {
    const float s = mm_logistic(1.f, kLog2e * z);
    slope = s * (1.f + z * (1.f - s));
    return z * s;
  }
  if (kAct == FS_ACT_GELU) {
    const float p = mm_phi(z);
    slope = p + z * 0.39894228f * ex2(-0.5f * kLog2e * z * z);
    return z * p;
  }
  if (kAct == FS_ACT_GELU_TANH) {
    const float s = mm_logistic(1.f, 2.f * kLog2e * kTanhC * (z + kTanhD * z * z * z));
    slope = s + z * s * (1.f - s) * 2.f * kTanhC * (1.f + 3.f * kTanhD * z * z);
    return z * s;
  }
  slope = 1.f;
  return z;
}

// f with the activation as a constant.
template <typename F>
__device__ __forceinline__ void mm_with_act(int act, F&& f) {
  switch (act) {
    case FS_ACT_RELU: f(std::integral_constant<int, FS_ACT_RELU>()); break;
    case FS_ACT_SILU: f(std::integral_constant<int, FS_ACT_SILU>()); break;
    case FS_ACT_GELU: f(std::integral_constant<int, FS_ACT_GELU>()); break;
    case FS_ACT_GELU_TANH: f(std::integral_constant<int, FS_ACT_GELU_TANH>()); break;
    default: f(std::integral_constant<int, FS_ACT_NONE>());
  }
}

}  // namespace fs
