// The products of a rank's layer: entry points, and rows to e4m3.
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <type_traits>

#include "fs_mm.cuh"

namespace fs {

int record_error(int code, const char* msg);

namespace {

int say(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return record_error(code, buf);
}

int cuda_say(cudaError_t e, const char* what) { return say(FS_ECUDA, "%s: %s", what, cudaGetErrorString(e)); }

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

constexpr int kMaxSize = 1 << 24;

int check_sizes(int rows, int in, int out) {
  if (rows < 0 || rows > kMaxSize) return say(FS_EINVAL, "rows = %d outside [0, 2^24]", rows);
  if (in < 1 || in > kMaxSize) return say(FS_EINVAL, "in = %d outside [1, 2^24]", in);
  if (out < 0 || out > kMaxSize) return say(FS_EINVAL, "out = %d outside [0, 2^24]", out);
  return FS_OK;
}

int check_types(int type, int out_type, int act) {
  if (type != FS_KV_BF16 && type != FS_KV_FP16 && type != FS_E4M3)
    return say(FS_EINVAL, "type = %d is not FS_KV_BF16, FS_KV_FP16 or FS_E4M3", type);
  if (out_type != FS_KV_BF16 && out_type != FS_KV_FP16) return say(FS_EINVAL, "out_type = %d is not FS_KV_BF16 or FS_KV_FP16", out_type);
  if (type != FS_E4M3 && out_type != type) return say(FS_EINVAL, "out_type = %d with operands of type %d", out_type, type);
  if (act < FS_ACT_NONE || act > FS_ACT_GELU_TANH) return say(FS_EINVAL, "activation = %d is none of FS_ACT_*", act);
  return FS_OK;
}

// Rows as the kernels may use them: the stride of a single row is one that any row could have.
int check_rows(fs_mm_rows& r, const char* name, int n, int width, int type, bool broadcast = false) {
  const int step = type == FS_E4M3 ? 16 : 8;
  if (n == 0) return FS_OK;
  if (!r.data) return say(FS_EINVAL, "%s is NULL", name);
  if (!aligned(r.data, 16)) return say(FS_EINVAL, "%s is not 16-byte aligned", name);
  if (n == 1) r.stride = (width + step - 1) / step * step;
  if (r.stride % step || (r.stride < width && !(broadcast && r.stride == 0)) || r.stride >= (1ll << 38))
    return say(FS_EINVAL, "%s: stride = %lld must be a multiple of %d elements, at least the width %d", name, (long long)r.stride, step, width);
  if ((type == FS_E4M3) != (r.scale != nullptr)) return say(FS_EINVAL, "%s: e4m3 codes have scales, other rows none", name);
  if (!aligned(r.scale, 16)) return say(FS_EINVAL, "%s: scales are not 16-byte aligned", name);
  return FS_OK;
}

constexpr int64_t kMmPartAt = 256;  // the status word, then dg and du of a backward pass

long long padded(int n) { return ((long long)n + 63) & ~63ll; }

int64_t workspace_of(int rows, int out, bool backward) { return kMmPartAt + (backward ? 4ll * rows * padded(out) : 0); }

int check_workspace(const void* ws, int64_t bytes, int64_t need) {
  if (!ws) return say(FS_EINVAL, "workspace is NULL");
  if (!aligned(ws, 256)) return say(FS_EINVAL, "workspace is not 256-byte aligned");
  if (bytes < need)
    return say(FS_EINVAL, "workspace of %lld bytes is less than the %lld this call needs", (long long)bytes, (long long)need);
  return FS_OK;
}

// Rows of an operand as boxes of `box_rows` rows and 128 bytes of them, swizzled.
int rows_map(CUtensorMap* m, const void* base, int n, int width, long long stride, int type, int box_rows) {
  const EncodeTiled enc = encode_tiled();
  if (!enc) return say(FS_ECUDA, "the driver has no cuTensorMapEncodeTiled");
  const int size = type == FS_E4M3 ? 1 : 2;
  const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)n}, strides[1] = {(cuuint64_t)stride * size};
  const cuuint32_t box[2] = {(cuuint32_t)(kMmBlock / size), (cuuint32_t)box_rows}, step[2] = {1, 1};
  const CUresult r = enc(m, size == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(base), dims, strides, box,
                         step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? FS_OK : say(FS_ECUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
}

// act(x W^T + bias) + residual, or with `up` the gated product, of few rows.
int few_product(const fs_mm_rows& x, const fs_mm_rows& w, const fs_mm_rows* up, const MmEpilogue& e, int in, int type, int out_type,
                uint32_t* status, cudaStream_t s, const char* what) {
  int dev = 0;
  const cudaError_t d = cudaGetDevice(&dev);
  if (d != cudaSuccess) return cuda_say(d, "cudaGetDevice");
  const int sms = sm_count_of(dev);
  if (!sms) return say(FS_ECUDA, "device query failed");
  const int per = kMmBlock / (type == FS_E4M3 ? 1 : 2), blocks = (in + per - 1) / per;
  const MmFewPlan p = mm_few_plan(e.rows, e.cols, blocks, up, sms);
  const int w_box = up ? p.w_rows / 2 : p.w_rows;
  CUtensorMap mx, mw, mu;
  if (int rc = rows_map(&mx, x.data, e.rows, in, x.stride, type, p.tokens)) return rc;
  if (int rc = rows_map(&mw, w.data, e.cols, in, w.stride, type, w_box)) return rc;
  if (up)
    if (int rc = rows_map(&mu, up->data, e.cols, in, up->stride, type, w_box)) return rc;
  const cudaError_t r = launch_mm_few(mx, mw, up ? &mu : nullptr, e, p, blocks, type, out_type, status, s);
  return r == cudaSuccess ? FS_OK : cuda_say(r, what);
}

// ---------------------------------------------------------------- products

// An operand: element (i, k) at data + i * i_step + k * k_step.
struct MmOperand {
  const void* data;
  long long i_step, k_step;
};

enum { MM_LINEAR, MM_GATED, MM_BACK };

struct MmArgs {
  MmOperand a[2], b[2];  // sums of MM_LINEAR run over a[0] b[0], then a[1] b[1]; MM_GATED, MM_BACK: a[0] with each b
  int inner[2];          // (of MM_LINEAR's second sum: 0 is none)
  int type;
  MmEpilogue e;
};

__device__ __forceinline__ float load_any(const MmOperand& o, int type, long long i, int k) {
  const long long at = i * o.i_step + k * o.k_step;
  if (type == FS_KV_BF16) return __uint_as_float((uint32_t) static_cast<const uint16_t*>(o.data)[at] << 16);
  if (type == FS_KV_FP16) return __half2float(static_cast<const __half*>(o.data)[at]);
  const uint32_t c = static_cast<const uint8_t*>(o.data)[at];
  const uint32_t h = e4m3x2_to_f16x2(c);
  return __half2float(__ushort_as_half((unsigned short)h));
}

// A tile of 64 x 64 results a block, 16 sums (of each product) a thread.
template <typename T, int kMode>
__global__ void __launch_bounds__(256) k_mm_simple(const MmArgs p) {
  constexpr int kB = kMode == MM_LINEAR ? 1 : 2;
  __shared__ float as[16][65], bs[kB][16][65];
  pdl_trigger();
  pdl_wait();
  const MmEpilogue& e = p.e;
  const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[kB][4][4] = {};
  for (int part = 0; part < (kMode == MM_LINEAR ? 2 : 1); ++part) {
    for (int k0 = 0; k0 < p.inner[part]; k0 += 16) {
      for (int i = threadIdx.x; i < 1024; i += 256) {
        const int r = i >> 4, k = i & 15;
        const bool in = k0 + k < p.inner[part];
        as[k][r] = in && m0 + r < e.rows ? load_any(p.a[part], p.type, m0 + r, k0 + k) : 0.f;
#pragma unroll
        for (int b = 0; b < kB; ++b) bs[b][k][r] = in && n0 + r < e.cols ? load_any(p.b[part + b], p.type, n0 + r, k0 + k) : 0.f;
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 16; ++k)
#pragma unroll
        for (int b = 0; b < kB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[b][i][j] = fmaf(as[k][ty * 4 + i], bs[b][k][tx * 4 + j], acc[b][i][j]);
      __syncthreads();
    }
  }
  mm_with_act(e.act, [&](auto act) {
    constexpr int kAct = decltype(act)::value;
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < 4; ++j) {
        const int m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
        if (m >= e.rows || n >= e.cols) continue;
        float z[2] = {acc[0][i][j], acc[kB - 1][i][j]};
        if (e.x_scale)
          for (int b = 0; b < kB; ++b) z[b] = z[b] * e.x_scale[m] * e.w_scale[b][n];
        T* out = static_cast<T*>(e.out[0]) + m * e.out_stride + n;
        const T* in = e.in ? static_cast<const T*>(e.in) + m * e.in_stride + n : nullptr;
        if (kMode == MM_LINEAR) {
          float y = z[0];
          if (e.bias) y += (float)static_cast<const T*>(e.bias)[n];
          y = mm_act<kAct>(y);
          if (in) y += (float)*in;
          *out = (T)y;
        } else if (kMode == MM_GATED) {
          *out = (T)(mm_act<kAct>(z[0]) * z[1]);
        } else {
          float slope;
          const float a = mm_act_slope<kAct>(z[0], slope), dy = (float)*in;
          *out = (T)(dy * z[1] * slope);
          static_cast<T*>(e.out[1])[m * e.out_stride + n] = (T)(dy * a);
        }
      }
  });
}

template <int kMode>
cudaError_t launch_mm(const MmArgs& p, int out_type, cudaStream_t s) {
  const dim3 grid((p.e.cols + 63) / 64, (p.e.rows + 63) / 64);
  return out_type == FS_KV_FP16 ? launch_pdl(k_mm_simple<__half, kMode>, grid, dim3(256), 0, s, p)
                                : launch_pdl(k_mm_simple<__nv_bfloat16, kMode>, grid, dim3(256), 0, s, p);
}

// ---------------------------------------------------------------- rows to e4m3

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// The least power of two s >= 2^-126 with amax <= 448 s; 0 for 0. amax finite.
__device__ __forceinline__ float scale_for(float amax) {
  if (!(amax > 0.f)) return 0.f;
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 127;
  return exp2_int(max(e - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0), -126));  // 448 = 1.75 * 2^8
}

template <typename T>
__global__ void __launch_bounds__(256) k_quantise_rows(int in, const T* x, long long x_stride, uint8_t* codes, long long c_stride, float* scale) {
  __shared__ float top[8];
  pdl_trigger();
  pdl_wait();
  const long long row = blockIdx.x;
  const T* xr = x + row * x_stride;
  uint8_t* cr = codes + row * c_stride;
  float amax = 0.f;
  for (int k = threadIdx.x; k < in; k += 256) {
    const float v = fabsf((float)xr[k]);
    if (v < INFINITY) amax = fmaxf(amax, v);
  }
  for (int o = 16; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, o));
  if ((threadIdx.x & 31) == 0) top[threadIdx.x >> 5] = amax;
  __syncthreads();
  for (int i = 0; i < 8; ++i) amax = fmaxf(amax, top[i]);
  const float s = scale_for(amax), inv = s > 0.f ? 1.f / s : 0.f;
  for (int k = threadIdx.x; k < in; k += 256) {
    const float v = (float)xr[k];
    cr[k] = fabsf(v) < INFINITY ? (uint8_t)e4m3x2(v * inv, 0.f) : 0x7f;
  }
  if (threadIdx.x == 0) scale[row] = s;
}

}  // namespace
}  // namespace fs

using namespace fs;

extern "C" int fs_mm_workspace_bytes(int32_t rows, int32_t in, int32_t out, int32_t backward, int64_t* bytes) {
  if (!bytes) return say(FS_EINVAL, "bytes is NULL");
  if (int rc = check_sizes(rows, in, out)) return rc;
  if (backward != 0 && backward != 1) return say(FS_EINVAL, "backward = %d is not 0 or 1", backward);
  *bytes = workspace_of(rows, out, backward);
  return FS_OK;
}

extern "C" int fs_linear(const fs_mm_linear* args, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  if (!args) return say(FS_EINVAL, "args is NULL");
  fs_mm_linear g = *args;
  if (int rc = check_sizes(g.rows, g.in, g.out)) return rc;
  if (int rc = check_types(g.type, g.out_type, g.activation)) return rc;
  if (int rc = check_workspace(workspace, workspace_bytes, kMmPartAt)) return rc;
  if (g.rows == 0 || g.out == 0) return FS_OK;
  if (int rc = check_rows(g.x, "x", g.rows, g.in, g.type)) return rc;
  if (int rc = check_rows(g.w, "w", g.out, g.in, g.type)) return rc;
  if (int rc = check_rows(g.y, "y", g.rows, g.out, g.out_type)) return rc;
  if (g.residual.data)
    if (int rc = check_rows(g.residual, "residual", g.rows, g.out, g.out_type, true)) return rc;
  if (!aligned(g.bias, 16)) return say(FS_EINVAL, "bias is not 16-byte aligned");
  MmArgs p{};
  p.a[0] = {g.x.data, g.x.stride, 1}, p.b[0] = {g.w.data, g.w.stride, 1};
  p.inner[0] = g.in, p.type = g.type;
  p.e = {g.rows, g.out, g.activation, g.x.scale, {g.w.scale, nullptr}, g.bias, g.residual.data, g.residual.stride, {g.y.data, nullptr}, g.y.stride};
  if (g.rows <= 1024)
    return few_product(g.x, g.w, nullptr, p.e, g.in, g.type, g.out_type, static_cast<uint32_t*>(workspace), static_cast<cudaStream_t>(cuda_stream),
                       "launch (fs_linear)");
  const cudaError_t e = launch_mm<MM_LINEAR>(p, g.out_type, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? FS_OK : cuda_say(e, "launch (fs_linear)");
}

extern "C" int fs_gated_ff(const fs_mm_gated* args, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  if (!args) return say(FS_EINVAL, "args is NULL");
  fs_mm_gated g = *args;
  if (int rc = check_sizes(g.rows, g.in, g.out)) return rc;
  if (int rc = check_types(g.type, g.out_type, g.activation)) return rc;
  if (int rc = check_workspace(workspace, workspace_bytes, kMmPartAt)) return rc;
  if (g.rows == 0 || g.out == 0) return FS_OK;
  if (int rc = check_rows(g.x, "x", g.rows, g.in, g.type)) return rc;
  if (int rc = check_rows(g.w_gate, "w_gate", g.out, g.in, g.type)) return rc;
  if (int rc = check_rows(g.w_up, "w_up", g.out, g.in, g.type)) return rc;
  if (int rc = check_rows(g.y, "y", g.rows, g.out, g.out_type)) return rc;
  MmArgs p{};
  p.a[0] = {g.x.data, g.x.stride, 1}, p.b[0] = {g.w_gate.data, g.w_gate.stride, 1}, p.b[1] = {g.w_up.data, g.w_up.stride, 1};
  p.inner[0] = g.in, p.type = g.type;
  p.e = {g.rows, g.out, g.activation, g.x.scale, {g.w_gate.scale, g.w_up.scale}, nullptr, nullptr, 0, {g.y.data, nullptr}, g.y.stride};
  if (g.rows <= 1024)
    return few_product(g.x, g.w_gate, &g.w_up, p.e, g.in, g.type, g.out_type, static_cast<uint32_t*>(workspace),
                       static_cast<cudaStream_t>(cuda_stream), "launch (fs_gated_ff)");
  const cudaError_t e = launch_mm<MM_GATED>(p, g.out_type, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? FS_OK : cuda_say(e, "launch (fs_gated_ff)");
}

extern "C" int fs_gated_ff_backward(const fs_mm_gated_grad* args, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  if (!args) return say(FS_EINVAL, "args is NULL");
  fs_mm_gated_grad g = *args;
  if (int rc = check_sizes(g.rows, g.in, g.out)) return rc;
  if (int rc = check_types(g.type, g.type, g.activation)) return rc;
  if (int rc = check_workspace(workspace, workspace_bytes, workspace_of(g.rows, g.out, true))) return rc;
  if (int rc = check_rows(g.x, "x", g.rows, g.in, g.type)) return rc;
  if (int rc = check_rows(g.w_gate, "w_gate", g.out, g.in, g.type)) return rc;
  if (int rc = check_rows(g.w_up, "w_up", g.out, g.in, g.type)) return rc;
  if (int rc = check_rows(g.dy, "dy", g.out ? g.rows : 0, g.out, g.type)) return rc;
  if (int rc = check_rows(g.dx, "dx", g.rows, g.in, g.type)) return rc;
  if (int rc = check_rows(g.dw_gate, "dw_gate", g.out, g.in, g.type)) return rc;
  if (int rc = check_rows(g.dw_up, "dw_up", g.out, g.in, g.type)) return rc;
  const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaSuccess;
  if (g.rows == 0 || g.out == 0) {  // sums over nothing
    auto clear = [&](const fs_mm_rows& r, int n) {
      if (n && e == cudaSuccess) e = cudaMemset2DAsync(r.data, 2 * r.stride, 0, 2 * (size_t)g.in, n, s);
    };
    clear(g.dx, g.rows), clear(g.dw_gate, g.out), clear(g.dw_up, g.out);
    return e == cudaSuccess ? FS_OK : cuda_say(e, "clear (fs_gated_ff_backward)");
  }
  const long long ld = padded(g.out);
  char* dg = static_cast<char*>(workspace) + kMmPartAt;
  char* du = dg + 2 * g.rows * ld;
  MmArgs p{};
  p.a[0] = {g.x.data, g.x.stride, 1}, p.b[0] = {g.w_gate.data, g.w_gate.stride, 1}, p.b[1] = {g.w_up.data, g.w_up.stride, 1};
  p.inner[0] = g.in, p.type = g.type;
  p.e = {g.rows, g.out, g.activation, nullptr, {}, nullptr, g.dy.data, g.dy.stride, {dg, du}, ld};
  e = launch_mm<MM_BACK>(p, g.type, s);
  if (e == cudaSuccess) {
    p.a[0] = {dg, ld, 1}, p.a[1] = {du, ld, 1}, p.b[0] = {g.w_gate.data, 1, g.w_gate.stride}, p.b[1] = {g.w_up.data, 1, g.w_up.stride};
    p.inner[0] = p.inner[1] = g.out;
    p.e = {g.rows, g.in, FS_ACT_NONE, nullptr, {}, nullptr, nullptr, 0, {g.dx.data, nullptr}, g.dx.stride};
    e = launch_mm<MM_LINEAR>(p, g.type, s);
  }
  for (int i = 0; i < 2 && e == cudaSuccess; ++i) {
    const fs_mm_rows& dw = i ? g.dw_up : g.dw_gate;
    p.a[0] = {i ? du : dg, 1, ld}, p.b[0] = {g.x.data, 1, g.x.stride};
    p.inner[0] = g.rows, p.inner[1] = 0;
    p.e = {g.out, g.in, FS_ACT_NONE, nullptr, {}, nullptr, nullptr, 0, {dw.data, nullptr}, dw.stride};
    e = launch_mm<MM_LINEAR>(p, g.type, s);
  }
  return e == cudaSuccess ? FS_OK : cuda_say(e, "launch (fs_gated_ff_backward)");
}

extern "C" int fs_quantise_rows(int32_t rows, int32_t in, int32_t type, const fs_mm_rows* x, const fs_mm_rows* codes, float* scale,
                                void* cuda_stream) {
  if (int rc = check_sizes(rows, in, 0)) return rc;
  if (type != FS_KV_BF16 && type != FS_KV_FP16) return say(FS_EINVAL, "type = %d is not FS_KV_BF16 or FS_KV_FP16", type);
  if (!x || !codes) return say(FS_EINVAL, "x / codes is NULL");
  if (rows == 0) return FS_OK;
  fs_mm_rows xr = *x, cr = *codes;
  cr.scale = scale;
  if (!scale) return say(FS_EINVAL, "scale is NULL");
  if (int rc = check_rows(xr, "x", rows, in, type)) return rc;
  if (int rc = check_rows(cr, "codes", rows, in, FS_E4M3)) return rc;
  const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = type == FS_KV_FP16
                            ? launch_pdl(k_quantise_rows<__half>, dim3(rows), dim3(256), 0, s, in, static_cast<const __half*>(xr.data),
                                         (long long)xr.stride, static_cast<uint8_t*>(cr.data), (long long)cr.stride, scale)
                            : launch_pdl(k_quantise_rows<__nv_bfloat16>, dim3(rows), dim3(256), 0, s, in, static_cast<const __nv_bfloat16*>(xr.data),
                                         (long long)xr.stride, static_cast<uint8_t*>(cr.data), (long long)cr.stride, scale);
  return e == cudaSuccess ? FS_OK : cuda_say(e, "launch (fs_quantise_rows)");
}

extern "C" int fs_mm_check(void* workspace, void* cuda_stream) {
  if (int rc = check_workspace(workspace, kMmPartAt, kMmPartAt)) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  uint32_t st = 0;
  cudaError_t e = cudaMemcpyAsync(&st, workspace, 4, cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) return cuda_say(e, "synchronize (fs_mm_check)");
  if (!st) return FS_OK;
  e = cudaMemsetAsync(workspace, 0, kMmPartAt, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) return cuda_say(e, "clear (fs_mm_check)");
  return say(FS_ETIMEOUT, "a device wait timed out (status 0x%x)", st);
}
