// The products of a rank's layer: entry points, and rows to e4m3.
#include <algorithm>
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <type_traits>
#include <utility>

#include "fs_mm.cuh"
#include "fs_rows_overlap.h"

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
constexpr int64_t kMaxElements = 1ll << 40;

int check_sizes(int rows, int in, int out) {
  if (rows < 0 || rows > kMaxSize) return say(FS_EINVAL, "rows = %d outside [0, 2^24]", rows);
  if (in < 1 || in > kMaxSize) return say(FS_EINVAL, "in = %d outside [1, 2^24]", in);
  if (out < 0 || out > kMaxSize) return say(FS_EINVAL, "out = %d outside [0, 2^24]", out);
  if (std::max({(int64_t)rows * in, (int64_t)rows * out, (int64_t)out * in}) >= kMaxElements)
    return say(FS_EINVAL, "rows = %d, in = %d, out = %d: an operand of 2^40 elements or more", rows, in, out);
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

// Whether two operands' rows share a byte.
struct Span {
  const fs_mm_rows* r;
  int n, width, size;  // rows, elements of a row, bytes of an element
  bool none() const { return !n || !width || !r->data; }
  // (a residual's rows may all be the same one)
  RowSpan rows() const { return {reinterpret_cast<int64_t>(r->data), r->stride ? n : 1, (int64_t)width * size, r->stride * size}; }
};
bool overlap(const Span& a, const Span& b) { return !a.none() && !b.none() && rows_overlap(a.rows(), b.rows()); }

// Outputs share nothing with inputs and each other.
int check_apart(const Span& out, const char* out_name, const Span& in, const char* in_name) {
  return overlap(out, in) ? say(FS_EINVAL, "%s and %s overlap", out_name, in_name) : FS_OK;
}
int check_apart(const Span& out, const char* out_name, const float* scales, int n, const char* in_name) {
  if (!scales) return FS_OK;
  const fs_mm_rows r{const_cast<float*>(scales), 0, nullptr};
  return overlap(out, {&r, 1, n, 4}) ? say(FS_EINVAL, "%s and the scales of %s overlap", out_name, in_name) : FS_OK;
}

constexpr int64_t kMmPartAt = 256;  // the status word, then dg and du of a backward pass, and what their rounding left

long long padded(int n) { return ((long long)n + 63) & ~63ll; }

int64_t workspace_of(int rows, int out, bool backward) { return kMmPartAt + (backward ? 2 * mm_terms(rows, out) : 0); }

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

constexpr int kFewRowsMost = 1024;  // (beyond, W would be read nine times and more)

// What every product needs of its call.
struct MmCall {
  int in, type, out_type, sms;
  uint32_t* status;
  cudaStream_t stream;
  const char* what;  // for errors
  int blocks() const { return (in + per() - 1) / per(); }
  int per() const { return kMmBlock / (type == FS_E4M3 ? 1 : 2); }
};

int device_sms(int* sms) {
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_say(e, "cudaGetDevice");
  *sms = sm_count_of(dev);
  return *sms ? FS_OK : say(FS_ECUDA, "device query failed");
}

// act(x W^T + bias) + residual, or with `up` the gated product, of few rows.
int few_product(const MmCall& c, const fs_mm_rows& x, const fs_mm_rows& w, const fs_mm_rows* up, const MmEpilogue& e, const MmFewPlan& p) {
  const int w_box = up ? p.w_rows / 2 : p.w_rows;
  CUtensorMap mx, mw, mu;
  if (int rc = rows_map(&mx, x.data, e.rows, c.in, x.stride, c.type, p.tokens)) return rc;
  if (int rc = rows_map(&mw, w.data, e.cols, c.in, w.stride, c.type, w_box)) return rc;
  if (up)
    if (int rc = rows_map(&mu, up->data, e.cols, c.in, up->stride, c.type, w_box)) return rc;
  const cudaError_t r = launch_mm_few(mx, mw, up ? &mu : nullptr, e, p, c.blocks(), c.type, c.out_type, c.status, c.stream);
  return r == cudaSuccess ? FS_OK : cuda_say(r, c.what);
}

// The same of many rows; with e.out[1] the first product of a backward pass, with e.out[2] in two terms.
int wide_product(const MmCall& c, const fs_mm_rows& x, const fs_mm_rows& w, const fs_mm_rows* up, const MmEpilogue& e, int tile) {
  MmWideArgs a{};
  if (int rc = rows_map(&a.maps[0], x.data, e.rows, c.in, x.stride, c.type, 128)) return rc;
  if (int rc = rows_map(&a.maps[1], w.data, e.cols, c.in, w.stride, c.type, tile / 2)) return rc;
  if (up)
    if (int rc = rows_map(&a.maps[2], up->data, e.cols, c.in, up->stride, c.type, tile / 2)) return rc;
  a.product[0] = {e, {0, 0}, {1, 2}, {c.blocks(), 0}, false, false, tile};
  a.products = 1;
  a.status = c.status;
  const cudaError_t r = launch_mm_wide(a, e.out[2] ? MM_BACK_TWO : e.out[1] ? MM_BACK : up ? MM_GATED : MM_LINEAR, c.type, c.out_type, c.sms, c.stream);
  return r == cudaSuccess ? FS_OK : cuda_say(r, c.what);
}

// By the kernel that the estimates say is faster.
int product(const MmCall& c, const fs_mm_rows& x, const fs_mm_rows& w, const fs_mm_rows* up, const MmEpilogue& e) {
  float ns = 0.f;
  const int tile = mm_wide_tile(e.rows, e.cols, c.blocks(), up, c.sms, &ns);
  if (e.rows <= kFewRowsMost) {
    const MmFewPlan p = mm_few_plan(e.rows, e.cols, c.blocks(), up, c.sms);
    if (p.ns < ns) return few_product(c, x, w, up, e, p);
  }
  return wide_product(c, x, w, up, e, tile);
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

// A row a group of kGroup threads (a warp of a block, or a block), eight values a thread at a time. Between the maximum and the codes a row is held: in registers,
// kHeld pieces a thread, or (kHeld = 0) in shared memory, where more rows an SM are under way at once; what it does not hold is read
// again. Bound by memory with many rows (8192 of 14336 bf16 54.6 us, 6.45 TB/s; with floats compared and every value looked at for
// what is not finite 72.7), by latency with few.
template <typename T, int kGroup, int kHeld>
__global__ void __launch_bounds__(kGroup == 32 ? 256 : kGroup) k_quantise_rows(int rows, int in, const T* x, long long x_stride, uint8_t* codes, long long c_stride, float* scale) {
  extern __shared__ uint4 row_at[];
  constexpr int kBlock = kGroup == 32 ? 256 : kGroup;
  __shared__ uint32_t top[8];
  pdl_trigger();
  pdl_wait();
  const long long row = (long long)blockIdx.x * (kBlock / kGroup) + threadIdx.x / kGroup;
  if (kGroup == 32 && row >= rows) return;
  const int id = threadIdx.x % kGroup, pieces = (in + 7) / 8;
  const T* xr = x + row * x_stride;
  uint8_t* cr = codes + row * c_stride;
  auto piece = [&](int p) {
    const uint16_t* at = reinterpret_cast<const uint16_t*>(xr) + 8 * p;
    if (8 * p + 8 <= in) return *reinterpret_cast<const uint4*>(at);
    uint32_t w[4] = {0, 0, 0, 0};
    for (int i = 0; 8 * p + i < in; ++i) w[i >> 1] |= (uint32_t)at[i] << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
  };
  // magnitudes are in the order of their bits: two at a time, and what is not finite above all others
  constexpr uint32_t kInf = std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;
  uint32_t most = 0;
  auto look = [&](uint4 u) {
    most = __vmaxu2(most, __vmaxu2(__vmaxu2(u.x & 0x7fff7fffu, u.y & 0x7fff7fffu), __vmaxu2(u.z & 0x7fff7fffu, u.w & 0x7fff7fffu)));
  };
  // (where a row holds such values: the others alone)
  auto finite = [&](uint4 u) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = w[i] & 0x7fffu, hi = w[i] >> 16 & 0x7fffu;
      most = __vmaxu2(most, (lo < kInf ? lo : 0u) | (hi < kInf ? hi << 16 : 0u));
    }
  };
  // the row's largest, of all of the group's threads
  auto join = [&] {
    uint32_t m = max(most & 0xffffu, most >> 16);
#pragma unroll
    for (int o = 16; o; o >>= 1) m = max(m, __shfl_xor_sync(~0u, m, o));
    if (kGroup > 32) {
      __syncthreads();  // (the last join's have been read)
      if ((threadIdx.x & 31) == 0) top[threadIdx.x >> 5] = m;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kGroup / 32; ++i) m = max(m, top[i]);
    }
    return m;
  };
  bool odd = false;  // something in the row is not finite
  auto store = [&](int p, uint4 u, float inv) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    uint32_t y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = Elem<T>::two(w[i]);
      y[i] = e4m3x2(v.x * inv, v.y * inv);
      if (odd) {
        if ((w[i] & 0x7fffu) >= kInf) y[i] = (y[i] & 0xff00u) | 0x7fu;
        if ((w[i] >> 16 & 0x7fffu) >= kInf) y[i] = (y[i] & 0xffu) | 0x7f00u;
      }
    }
    const uint2 c = make_uint2(y[0] | y[1] << 16, y[2] | y[3] << 16);
    if (8 * p + 8 <= in) {
      *reinterpret_cast<uint2*>(cr + 8 * p) = c;
    } else {
      for (int i = 0; 8 * p + i < in; ++i) cr[8 * p + i] = (uint8_t)((i < 4 ? c.x >> (8 * i) : c.y >> (8 * (i - 4))) & 255u);
    }
  };
  constexpr int kRegs = kHeld ? kHeld : 1;
  uint4 held[kRegs];
  if (kHeld) {
#pragma unroll
    for (int j = 0; j < kRegs; ++j) held[j] = id + j * kGroup < pieces ? piece(id + j * kGroup) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < kRegs; ++j) look(held[j]);
    for (int p = id + kHeld * kGroup; p < pieces; p += kGroup) look(piece(p));
  } else {
    for (int p = id; p < pieces; p += kGroup) {  // (each thread reads back what it copied)
      if (8 * p + 8 <= in)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(row_at + p)), "l"(xr + 8 * p) : "memory");
      else
        row_at[p] = piece(p);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    for (int p = id; p < pieces; p += kGroup) look(row_at[p]);
  }
  uint32_t m = join();
  odd = m >= kInf;
  if (odd) {
    most = 0;
    if (kHeld) {
#pragma unroll
      for (int j = 0; j < kRegs; ++j) finite(held[j]);
      for (int p = id + kHeld * kGroup; p < pieces; p += kGroup) finite(piece(p));
    } else {
      for (int p = id; p < pieces; p += kGroup) finite(row_at[p]);
    }
    m = join();
  }
  const float amax = Elem<T>::two(m).x;
  const float s = scale_for(amax), inv = s > 0.f ? 1.f / s : 0.f;  // (a power of two: exact; 2^126 at most)
  if (kHeld) {
#pragma unroll
    for (int j = 0; j < kRegs; ++j)
      if (id + j * kGroup < pieces) store(id + j * kGroup, held[j], inv);
    for (int p = id + kHeld * kGroup; p < pieces; p += kGroup) store(p, piece(p), inv);
  } else {
    for (int p = id; p < pieces; p += kGroup) store(p, row_at[p], inv);
  }
  if (id == 0) scale[row] = s;
}

template <typename T>
cudaError_t launch_quantise(int rows, int in, const fs_mm_rows& x, const fs_mm_rows& codes, float* scale, cudaStream_t s) {
  const T* xd = static_cast<const T*>(x.data);
  uint8_t* cd = static_cast<uint8_t*>(codes.data);
  const long long xs = x.stride, cs = codes.stride;
  // Registers while all rows are under way at once, and where they hold a long row (64 rows of 8192 2.0 us in graphs, in shared memory 2.4;
  // 1300 of 4096 5.5, in shared memory 6.2; one of 2048 1.4, by a warp 2.8)
  if (in <= 8192 && (in > 6144 || rows <= (in <= 2048 ? 256 : 1536)))
    return launch_pdl(k_quantise_rows<T, 256, 4>, dim3(rows), dim3(256), 0, s, rows, in, xd, xs, cd, cs, scale);
  // many short rows: a warp each (4096 of 512 3.4, by blocks 4.6; 2048 of them 3.2 and 3.2)
  if (in <= 2048 && rows > 2048) return launch_pdl(k_quantise_rows<T, 32, 8>, dim3((rows + 7) / 8), dim3(256), 0, s, rows, in, xd, xs, cd, cs, scale);
  // else in what shared memory a block has without asking for more: blocks of 128 threads, so that more rows an SM are under way (8192 of 4096
  // 18.1, 256 threads 22.9; 8192 of 8192 32.2, 256 threads in registers 31.6), of 256 for longer ones (8192 of 14336 54.0, 128 threads 58.3,
  // in registers 65.5)
  const size_t row = (in + 7) / 8 * 16;
  if (in <= 6144) return launch_pdl(k_quantise_rows<T, 128, 0>, dim3(rows), dim3(128), row, s, rows, in, xd, xs, cd, cs, scale);
  if (rows > 256 && in <= 24000) return launch_pdl(k_quantise_rows<T, 256, 0>, dim3(rows), dim3(256), row, s, rows, in, xd, xs, cd, cs, scale);
  return launch_pdl(k_quantise_rows<T, 256, 8>, dim3(rows), dim3(256), 0, s, rows, in, xd, xs, cd, cs, scale);
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
  const int size = g.type == FS_E4M3 ? 1 : 2;
  const Span y{&g.y, g.rows, g.out, 2}, r{&g.residual, g.rows, g.out, 2};
  const fs_mm_rows bias{const_cast<void*>(g.bias), 0, nullptr};
  if (int rc = check_apart(y, "y", {&g.x, g.rows, g.in, size}, "x")) return rc;
  if (int rc = check_apart(y, "y", {&g.w, g.out, g.in, size}, "w")) return rc;
  if (int rc = check_apart(y, "y", g.x.scale, g.rows, "x")) return rc;
  if (int rc = check_apart(y, "y", g.w.scale, g.out, "w")) return rc;
  if (int rc = check_apart(y, "y", {&bias, 1, g.out, 2}, "bias")) return rc;
  if (g.residual.data != g.y.data || g.residual.stride != g.y.stride)
    if (int rc = check_apart(y, "y", r, "residual")) return rc;
  MmCall c{g.in, g.type, g.out_type, 0, static_cast<uint32_t*>(workspace), static_cast<cudaStream_t>(cuda_stream), "launch (fs_linear)"};
  if (int rc = device_sms(&c.sms)) return rc;
  return product(c, g.x, g.w, nullptr,
                 {g.rows, g.out, g.activation, g.x.scale, {g.w.scale, nullptr}, g.bias, g.residual.data, g.residual.stride, {g.y.data, nullptr}, g.y.stride});
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
  const int size = g.type == FS_E4M3 ? 1 : 2;
  const Span y{&g.y, g.rows, g.out, 2};
  if (int rc = check_apart(y, "y", {&g.x, g.rows, g.in, size}, "x")) return rc;
  if (int rc = check_apart(y, "y", {&g.w_gate, g.out, g.in, size}, "w_gate")) return rc;
  if (int rc = check_apart(y, "y", {&g.w_up, g.out, g.in, size}, "w_up")) return rc;
  if (int rc = check_apart(y, "y", g.x.scale, g.rows, "x")) return rc;
  if (int rc = check_apart(y, "y", g.w_gate.scale, g.out, "w_gate")) return rc;
  if (int rc = check_apart(y, "y", g.w_up.scale, g.out, "w_up")) return rc;
  MmCall c{g.in, g.type, g.out_type, 0, static_cast<uint32_t*>(workspace), static_cast<cudaStream_t>(cuda_stream), "launch (fs_gated_ff)"};
  if (int rc = device_sms(&c.sms)) return rc;
  return product(c, g.x, g.w_gate, &g.w_up,
                 {g.rows, g.out, g.activation, g.x.scale, {g.w_gate.scale, g.w_up.scale}, nullptr, nullptr, 0, {g.y.data, nullptr}, g.y.stride});
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
  const Span all[] = {{&g.dx, g.rows, g.in, 2}, {&g.dw_gate, g.out, g.in, 2}, {&g.dw_up, g.out, g.in, 2}, {&g.x, g.rows, g.in, 2},
                      {&g.w_gate, g.out, g.in, 2}, {&g.w_up, g.out, g.in, 2}, {&g.dy, g.rows, g.out, 2}};
  const char* const names[] = {"dx", "dw_gate", "dw_up", "x", "w_gate", "w_up", "dy"};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 7; ++j)
      if (int rc = check_apart(all[i], names[i], all[j], names[j])) return rc;
  MmCall c{g.in, g.type, g.type, 0, static_cast<uint32_t*>(workspace), static_cast<cudaStream_t>(cuda_stream), "launch (fs_gated_ff_backward)"};
  if (g.rows == 0 || g.out == 0) {  // sums over nothing
    cudaError_t e = cudaSuccess;
    auto clear = [&](const fs_mm_rows& r, int n) {
      if (n && e == cudaSuccess) e = cudaMemset2DAsync(r.data, 2 * r.stride, 0, 2 * (size_t)g.in, n, c.stream);
    };
    clear(g.dx, g.rows), clear(g.dw_gate, g.out), clear(g.dw_up, g.out);
    return e == cudaSuccess ? FS_OK : cuda_say(e, "clear (fs_gated_ff_backward)");
  }
  if (int rc = device_sms(&c.sms)) return rc;
  // dg and du, then everything that is made of them in one launch. They are rounded to the operands' type in between, as both operands of a
  // tensor-core product have one: as floats they could be read only by products of tf32, with W and x twice as long and at half the rate. With
  // the results' own rounding that is 1.4 times the error of one (bf16 2.3e-3 of 64 bits' results, 1.7e-3 in one rounding), in short sums more:
  // those have them in two terms (mm_two_terms_dw, mm_two_terms_dx). A half's range bounds them.
  const long long ld = padded(g.out);
  char* dg = static_cast<char*>(workspace) + kMmPartAt;
  char* du = dg + 2 * g.rows * ld;
  const bool dx_two = mm_two_terms_dx(g.out), dw_two = mm_two_terms_dw(g.rows), two = dx_two || dw_two;
  char* dg_left = two ? du + 2 * g.rows * ld : nullptr;
  char* du_left = two ? dg_left + 2 * g.rows * ld : nullptr;
  float ns = 0.f;
  if (int rc = wide_product(c, g.x, g.w_gate, &g.w_up, {g.rows, g.out, g.activation, nullptr, {}, nullptr, g.dy.data, g.dy.stride, {dg, du, dg_left, du_left}, ld},
                            mm_wide_tile(g.rows, g.out, c.blocks(), true, c.sms, &ns)))
    return rc;
  MmWideArgs a{};
  enum { DG, DU, DG_LEFT, DU_LEFT, WG_T, WU_T, DG_T, DU_T, DG_LEFT_T, DU_LEFT_T, X_T };
  const std::pair<int, const char*> terms[] = {{DG, dg}, {DU, du}, {DG_LEFT, dg_left}, {DU_LEFT, du_left}};
  for (const auto& [at, data] : terms) {
    if (!data) continue;
    if (int rc = rows_map(&a.maps[at], data, g.rows, g.out, ld, g.type, 128)) return rc;
    if (int rc = rows_map(&a.maps[at + DG_T - DG], data, g.rows, g.out, ld, g.type, 64)) return rc;
  }
  if (int rc = rows_map(&a.maps[WG_T], g.w_gate.data, g.out, g.in, g.w_gate.stride, g.type, 64)) return rc;
  if (int rc = rows_map(&a.maps[WU_T], g.w_up.data, g.out, g.in, g.w_up.stride, g.type, 64)) return rc;
  if (int rc = rows_map(&a.maps[X_T], g.x.data, g.rows, g.in, g.x.stride, g.type, 64)) return rc;
  auto to = [&](const fs_mm_rows& r, int n) { return MmEpilogue{n, g.in, FS_ACT_NONE, nullptr, {}, nullptr, nullptr, 0, {r.data, nullptr}, r.stride}; };
  const int out_blocks = (g.out + 63) / 64, row_blocks = (g.rows + 63) / 64;
  const int out_left = dx_two ? out_blocks : 0, row_left = dw_two ? row_blocks : 0;
  a.product[0] = {to(g.dx, g.rows), {DG, DU, DG_LEFT, DU_LEFT}, {WG_T, WU_T, WG_T, WU_T}, {out_blocks, out_blocks, out_left, out_left}, false, true};
  a.product[1] = {to(g.dw_gate, g.out), {DG_T, DG_LEFT_T}, {X_T, X_T}, {row_blocks, row_left}, true, true};
  a.product[2] = {to(g.dw_up, g.out), {DU_T, DU_LEFT_T}, {X_T, X_T}, {row_blocks, row_left}, true, true};
  a.products = 3;
  a.status = c.status;
  const cudaError_t e = launch_mm_wide(a, MM_GRAD, g.type, g.type, c.sms, c.stream);
  return e == cudaSuccess ? FS_OK : cuda_say(e, c.what);
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
  if (int rc = check_apart({&cr, rows, in, 1}, "codes", {&xr, rows, in, 2}, "x")) return rc;
  if (int rc = check_apart({&cr, rows, in, 1}, "codes", scale, rows, "codes")) return rc;
  if (int rc = check_apart({&xr, rows, in, 2}, "x", scale, rows, "codes")) return rc;
  const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = type == FS_KV_FP16 ? launch_quantise<__half>(rows, in, xr, cr, scale, s) : launch_quantise<__nv_bfloat16>(rows, in, xr, cr, scale, s);
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
