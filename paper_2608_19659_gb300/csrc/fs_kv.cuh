// Shared parts of the cache operators (fs_kv.cu, fs_kv_decode.cu, fs_kv_chunk.cu).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>

#include "fs_internal.cuh"

namespace fs {

// Bits of a cache workspace's status word besides ST_TIMEOUT.
enum : uint32_t {
  KV_ST_PAGE = 0x100u,    // a page id outside the cache
  KV_ST_BATCH = 0x200u,   // q_start or length out of order, or beyond the batch's bounds
  KV_ST_VALUE = 0x400u,   // a NaN among the keys or values of an append (stored as 0)
  KV_ST_ANGLE = 0x800u,   // a position beyond the rows of cos / sin
  KV_ST_SCALE = 0x1000u,  // a scale that is neither a power of two nor 0
};

// The workspace: status word, tickets (zero between calls), partial results.
constexpr int kKvTickets = 8192;
constexpr int kKvFan = 16;  // results that are joined at a time
constexpr int kKvCluster = 8;
constexpr size_t kKvTicketAt = 256;
constexpr size_t kKvPartAt = kKvTicketAt + 4 * (size_t)kKvTickets;

// What every kernel reads of the cache and the batch.
struct KvView {
  int pages, heads, log_page, batch, tokens, max_new, max_length, table_stride, group;  // group: query heads per key head
  const float *k_scale, *v_scale;
  const int *page_table, *length, *q_start;
  uint32_t* status;
};

struct KvAttendArgs {
  KvView v;
  const void* q;
  void* out;
  long long q_token, q_head, out_token, out_head;  // strides, elements
  float scale_log2;  // scale * log2(e)
  int window;        // 0: none
  int split;         // tokens per part of the cache axis
  int min_rows, max_rows;  // sequences with rows outside (min_rows, max_rows] are another kernel's
  float* part;       // partial results
  char* wide;        // k_kv_chunk: the walked tokens as halves (k_kv_expand), or null
  int wide_tiles;    // tiles of 128 tokens there, of a sequence
  unsigned* ticket;
  int cluster;       // blocks of a cluster: consecutive parts of one item
  int tickets;       // of an item: 1, or 1 and one for every kKvFan clusters
};

// One sequence of the batch as a kernel may use it: ranges checked, so that no
// later index leaves its array whatever the batch's device arrays hold (the host has
// checked that a page table's row holds max_length tokens).
struct KvSeq {
  int len, first, count;  // tokens cached, first row of q, rows of q
};

__device__ __forceinline__ bool kv_seq(const KvView& v, int b, KvSeq& s) {
  s.len = v.length[b];
  s.first = v.q_start[b];
  s.count = v.q_start[b + 1] - s.first;
  const bool ok = s.len >= 0 && s.len <= v.max_length && s.first >= 0 && s.count >= 0 && s.count <= v.max_new && s.first <= v.tokens - s.count;
  return ok;
}

__device__ __forceinline__ void kv_flag(const KvView& v, uint32_t bit) { atomicOr(v.status, bit); }

// Reports rows of the call that are no sequence's: before the first one's, or after the last one's.
__device__ __forceinline__ void kv_ends(const KvView& v, int b, const KvSeq& s) {
  if ((b == 0 && s.first != 0) || (b == v.batch - 1 && s.first + s.count != v.tokens)) kv_flag(v, KV_ST_BATCH);
}

// Page id `i` of sequence b. What writes to a page asks kv_page_held first and stores nothing
// where the table holds none of the cache's pages; reads take page 0 in its place (kv_page_ok). Both
// flag it. The check waits for the load: kv_page_raw apart lets other work come between.
__device__ __forceinline__ int kv_page_raw(const KvView& v, int b, int i) {
  return v.page_table[(long long)b * v.table_stride + i];
}
__device__ __forceinline__ bool kv_page_held(const KvView& v, int g) {
  if ((unsigned)g < (unsigned)v.pages) return true;
  kv_flag(v, KV_ST_PAGE);
  return false;
}
__device__ __forceinline__ int kv_page_ok(const KvView& v, int g) { return kv_page_held(v, g) ? g : 0; }
__device__ __forceinline__ int kv_page(const KvView& v, int b, int i) { return kv_page_ok(v, kv_page_raw(v, b, i)); }

// Scales are powers of two or 0, so that a code times a quotient of scales is exact in
// half precision; others are reported.
__device__ __forceinline__ bool kv_scale_ok(float s) {
  const uint32_t x = __float_as_uint(s);
  return x == 0 || ((x & 0x807fffffu) == 0 && x != 0x7f800000u);
}
__device__ __forceinline__ void kv_scales(const KvView& v, float ks, float vs) {
  if (!kv_scale_ok(ks) || !kv_scale_ok(vs)) kv_flag(v, KV_ST_SCALE);
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two e4m3 codes (the low or high half of w) as two halves; exact.
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t w) {
  uint32_t r;
  asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %1;\n cvt.rn.f16x2.e4m3x2 %0, lo;\n}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2_hi(uint32_t w) {
  uint32_t r;
  asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %1;\n cvt.rn.f16x2.e4m3x2 %0, hi;\n}" : "=r"(r) : "r"(w));
  return r;
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// One tile of the cache into shared memory: from token slot `token` of (page, head) on.
__device__ __forceinline__ void tma_tile(uint32_t dst, const CUtensorMap* m, int token, int head, int page, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(m), "r"(0), "r"(token), "r"(head), "r"(page), "r"(smem_u32(bar))
      : "memory");
}

template <typename T>
struct Elem;
template <>
struct Elem<__nv_bfloat16> {
  static __device__ __forceinline__ float2 two(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
  }
};
template <>
struct Elem<__half> {
  static __device__ __forceinline__ float2 two(uint32_t w) {
    __half2 h;
    memcpy(&h, &w, 4);
    return __half22float2(h);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack_f16(a, b); }
};

// A row's power of two: 2^-e with e the exponent of its largest magnitude, so that the
// row times it lies in [-2, 2] and rounds to half precision without overflow. (A bf16
// row's values keep their 8 bits there unless they are under 2^-14 of its largest.)
__device__ __forceinline__ int row_exponent(float amax) {
  const int e = (int)((__float_as_uint(amax) >> 23) & 255u) - 127;
  return min(max(e, -126), 126);
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126..127

// Raises a kernel's shared memory limit once on each device (seen: a bit a device, one word a kernel).
inline cudaError_t smem_limit_once(std::atomic<uint64_t>& seen, const void* kernel, size_t bytes) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (seen.load(std::memory_order_acquire) & bit) return cudaSuccess;
  e = raise_smem_limit(kernel, bytes);
  if (e == cudaSuccess && dev < 64) seen.fetch_or(bit, std::memory_order_release);
  return e;
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled();  // null: the driver has none
int sm_count_of(int dev);    // 0: not known

// A tensor map of a cache tensor: [pages][heads][page tokens][dim] bytes in tiles of
// `rows` tokens of one (page, head), its 16-byte pieces swizzled over the rows or in order.
int kv_tensor_map(CUtensorMap* m, const fs_kv_cache& c, const void* base, int rows, bool swizzled);

cudaError_t launch_kv_decode(const CUtensorMap& mk, const CUtensorMap& mv, const KvAttendArgs& a, int dim, int dtype,
                             int row_tile, int row_blocks, int splits, cudaStream_t s);
constexpr int kKvChunkRows = 256;  // rows of a block
cudaError_t launch_kv_chunk(const CUtensorMap& mk, const CUtensorMap& mv, const KvAttendArgs& a, const fs_kv_cache& c,
                            int dtype, int tiles, int parts, cudaStream_t s);

}  // namespace fs
