// Shared parts of the products of a rank's layer (fs_mm.cu and its kernels).
#pragma once

#include <type_traits>

#include "fs_kv.cuh"
#include "fs_mm_plan.h"
#include "fs_tc.cuh"

namespace fs {

// What a product's epilogue reads and writes. Rows are the call's rows (tokens), columns what W's rows are.
struct MmEpilogue {
  int rows, cols, act;
  const float* x_scale;     // e4m3: of each row, else null
  const float* w_scale[2];  // of each column (of gate and up)
  const void* bias;
  const void* in;  // residual, or dy of the backward pass
  long long in_stride;
  void* out[4];  // y; dg and du in the backward pass, and in two terms what their rounding left
  long long out_stride;
};

// A row's scale xs as near * far, for sums of e4m3 products (0, or 2^-18 to 2^42) that are multiplied by it and by a column's scale s, any
// floats: far is 2^64 or 2^-64 where xs itself would carry a sum out of a float's range that s brings back, else 1.
struct MmScale {
  float near, far;
};
__device__ __forceinline__ MmScale mm_scale(float xs) {
  const float m = fabsf(xs);
  if (m >= 0x1p60f) return {xs * 0x1p-64f, 0x1p64f};
  if (m <= 0x1p-60f && m > 0.f) return {xs * 0x1p64f, 0x1p-64f};  // (exact, of subnormals too)
  return {xs, 1.f};
}
// v[i] = (v[i] near) s[i] far, far where it keeps what is between in range: with s if it brings that nearer to 1, else last.
template <int n>
__device__ __forceinline__ void mm_scaled(float (&v)[n], MmScale x, const float (&s)[n]) {
  if (__builtin_expect(x.far == 1.f, 1)) {
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = v[i] * x.near * s[i];
  } else {
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = (fabsf(s[i]) < 1.f) == (x.far > 1.f) ? v[i] * x.near * (s[i] * x.far) : v[i] * x.near * s[i] * x.far;
  }
}

// z / (1 + e^-2h), 2 log2(e) h in `e`: the logistic function's share of z. The quotient is
// off by 2 ulp, and 0 where e^-2h passes 2^126 (values under 2^-119 of z).
__device__ __forceinline__ float mm_logistic(float z, float e) { return __fdividef(z, 1.f + ex2(-e)); }

constexpr float kLog2e = 1.44269504f, kTanhC = 0.7978845608f, kTanhD = 0.044715f;

// Phi(z): without cancellation in the lower tail, as e^(-z^2 / 2) t P(t), t = 1 / (1 + 0.45 |z| / sqrt 2). t P(t) stands for half of
// e^(x^2) erfc(x), x = |z| / sqrt 2, which falls as t does; P is of degree 7, fitted to it over x <= 10.5 for the least largest relative
// error (Lawson's reweighted least squares): 3.2e-7, 7e-7 with the roundings, of the exponential z^2 2^-24 besides. (4096 rows of 512
// over 4096 columns: 53 us by the library's erfcf, whose instructions were five times these.)
__device__ __forceinline__ float mm_phi(float z) {
  const float t = __fdividef(1.f, 1.f + 0.31819806f * fabsf(z));
  float p = 0.03364478f;
  p = p * t - 0.12102614f;
  p = p * t + 0.10597738f;
  p = p * t + 0.018687509f;
  p = p * t + 0.09511253f;
  p = p * t + 0.113793775f;
  p = p * t + 0.12685856f;
  p = p * t + 0.12695177f;
  p *= t * ex2(-0.5f * kLog2e * z * z);
  return z < 0.f ? p : 1.f - p;
}

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
    // (beyond |z| = 20 s is 0 or 1, and z^2 may overflow)
    slope = s + z * s * (1.f - s) * 2.f * kTanhC * (1.f + 3.f * kTanhD * fminf(z * z, 400.f));
    return z * s;
  }
  slope = 1.f;
  return z;
}

// Four neighbouring 16-bit values of a row, n of them inside it (others 0; all when n >= 4: then 8 bytes at once).
__device__ __forceinline__ uint2 mm_raw4(const uint16_t* p, int n) {
  if (n >= 4) return *reinterpret_cast<const uint2*>(p);
  uint2 v = make_uint2(0, 0);
  if (n > 0) v.x = p[0];
  if (n > 1) v.x |= (uint32_t)p[1] << 16;
  if (n > 2) v.y = p[2];
  return v;
}
template <typename T>
__device__ __forceinline__ float4 mm_floats4(uint2 w) {
  const float2 a = Elem<T>::two(w.x), b = Elem<T>::two(w.y);
  return make_float4(a.x, a.y, b.x, b.y);
}
template <typename T>
__device__ __forceinline__ void mm_store4(T* p, float4 v, int n) {
  if (n >= 4) {
    *reinterpret_cast<uint2*>(p) = make_uint2(Elem<T>::pack(v.x, v.y), Elem<T>::pack(v.z, v.w));
    return;
  }
  if (n > 0) p[0] = (T)v.x;
  if (n > 1) p[1] = (T)v.y;
  if (n > 2) p[2] = (T)v.z;
}
__device__ __forceinline__ float4 mm_load4(const float* p, int n) {
  if (n >= 4) return *reinterpret_cast<const float4*>(p);
  return make_float4(n > 0 ? p[0] : 0.f, n > 1 ? p[1] : 0.f, n > 2 ? p[2] : 0.f, 0.f);
}
__device__ __forceinline__ float4 mm_scaled(float4 v, MmScale x, float4 s) {
  float a[4] = {v.x, v.y, v.z, v.w};
  mm_scaled(a, x, {s.x, s.y, s.z, s.w});
  return make_float4(a[0], a[1], a[2], a[3]);
}
__device__ __forceinline__ float4 operator*(float4 a, float b) { return make_float4(a.x * b, a.y * b, a.z * b, a.w * b); }
__device__ __forceinline__ float4 operator*(float4 a, float4 b) { return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w); }
__device__ __forceinline__ float4 operator+(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }

// What kernels ahead stored, for the copies of this thread.
__device__ __forceinline__ void fence_proxy_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }

// A box of rows into shared memory: from element `x` of row `y` on.
__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap* m, int x, int y, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"(m), "r"(x), "r"(y), "r"(smem_u32(bar))
               : "memory");
}

// A whole warp's wait, which says so when it runs out; the caller leaves its loop. Every thread gives up by its own clock, but the
// answer is the warp's: what it guards are instructions of whole warps (tcgen05.ld, barriers).
__device__ __forceinline__ bool mm_wait(uint64_t* bar, uint32_t parity, uint32_t* status) {
  const bool ok = mbar_wait(bar, parity, kWaitLimitNs);
  if (!ok) atomicOr(status, ST_TIMEOUT);
  return __all_sync(~0u, ok);
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

// x and one or two W, each in boxes of one block and the plan's rows.
cudaError_t launch_mm_few(const CUtensorMap& x, const CUtensorMap& w, const CUtensorMap* up, const MmEpilogue& e, const MmFewPlan& p,
                          int blocks_k, int type, int out_type, uint32_t* status, cudaStream_t s);

enum { MM_LINEAR, MM_GATED, MM_BACK, MM_GRAD, MM_BACK_TWO };

// One product of a launch of k_mm_wide: e.rows x e.cols results, sums over blocks[0] blocks of maps a[0] and b[0] (MM_GATED, MM_BACK, MM_BACK_TWO:
// b[0] for gate and b[1] for up). Maps have boxes of 128 rows (B: half a tile's columns) and one block. MM_GRAD: up to three products,
// whose sums go on over blocks[i] blocks of a[i] and b[i], and whose operands may lie the other way (a_mn, b_mn: the rows are
// contiguous, boxes are of 64 of them and 64 terms of the sum); results are stored as they are.
struct MmProduct {
  MmEpilogue e;
  int a[4], b[4], blocks[4];
  bool a_mn, b_mn;
  int tile;         // (MM_GRAD: launch_mm_wide's) columns of a tile (gated: of gate and of up together): a multiple of 32 (gated: 64) up to 256
  // launch_mm_wide's: tiles of rows, tiles in all, and of a group of rows' tiles that are walked over together. (Under 2^31: no operand
  // has 2^40 elements)
  int row_tiles, tiles, group;
};
struct MmWideArgs {
  CUtensorMap maps[11];
  MmProduct product[3];
  int products, eight, format;
  int lead, rounds;        // (launch_mm_wide's: pairs that start with one of the longest tiles, and how many others that takes as long as)
  int stages, stage, sub;  // (launch_mm_wide's: stages of the ring, their bytes, and blocks of the sum)
  int tiles;
  uint32_t* status;
};
cudaError_t launch_mm_wide(MmWideArgs& a, int mode, int type, int out_type, int sms, cudaStream_t s);

}  // namespace fs
