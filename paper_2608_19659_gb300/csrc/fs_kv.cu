// The cache operators' entry points, and appending to the cache.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "fs_kv.cuh"

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

int log2_page(int p) { return p == 16 ? 4 : p == 32 ? 5 : p == 64 ? 6 : p == 128 ? 7 : -1; }

int check_cache(const fs_kv_cache* c) {
  if (!c) return say(FS_EINVAL, "cache is NULL");
  if (c->pages < 1) return say(FS_EINVAL, "cache pages = %d < 1", c->pages);
  if (c->heads < 1 || c->heads > 1024) return say(FS_EINVAL, "cache heads = %d outside [1, 1024]", c->heads);
  if (log2_page(c->page_tokens) < 0) return say(FS_EINVAL, "page_tokens = %d is not 16, 32, 64 or 128", c->page_tokens);
  if (c->dim != 64 && c->dim != 128) return say(FS_EINVAL, "dim = %d is not 64 or 128", c->dim);
  if (!c->k || !c->v || !c->k_scale || !c->v_scale) return say(FS_EINVAL, "a cache pointer is NULL");
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return say(FS_EINVAL, "cache k / v are not 16-byte aligned");
  if (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return say(FS_EINVAL, "cache scales are not 4-byte aligned");
  const int64_t st[3] = {c->page_stride, c->head_stride, c->token_stride};
  for (int64_t s : st)
    if (s < 16 || s % 16 || s >= (1ll << 40)) return say(FS_EINVAL, "cache strides must be multiples of 16 in [16, 2^40)");
  if (c->token_stride < c->dim) return say(FS_EINVAL, "cache token_stride is less than dim");
  return FS_OK;
}

int check_batch(const fs_kv_cache* c, const fs_kv_batch* b, int q_heads) {
  if (!b) return say(FS_EINVAL, "batch is NULL");
  if (b->batch < 0 || b->batch > 65535) return say(FS_EINVAL, "batch = %d outside [0, 65535]", b->batch);
  if (b->tokens < 0 || b->max_new < 0 || b->max_new > b->tokens)
    return say(FS_EINVAL, "tokens = %d, max_new = %d: want 0 <= max_new <= tokens", b->tokens, b->max_new);
  if (b->batch && (int64_t)b->batch * b->max_new < b->tokens)
    return say(FS_EINVAL, "tokens = %d are more than batch * max_new = %d * %d", b->tokens, b->batch, b->max_new);
  if (b->max_length < 0 || b->max_length > (1 << 30))
    return say(FS_EINVAL, "max_length = %d outside [0, 2^30]", b->max_length);
  if (b->table_stride < 0 || (int64_t)b->table_stride * c->page_tokens < b->max_length)
    return say(FS_EINVAL, "table_stride = %d pages are fewer than max_length = %d tokens need", b->table_stride,
               b->max_length);
  if ((int64_t)b->table_stride * c->page_tokens > INT_MAX - 128) return say(FS_EINVAL, "table_stride = %d is too large", b->table_stride);
  if (q_heads < 1 || q_heads > 65535) return say(FS_EINVAL, "q_heads = %d outside [1, 65535]", q_heads);
  if ((int64_t)b->tokens * q_heads > (1 << 30)) return say(FS_EINVAL, "tokens * q_heads exceeds 2^30");
  if (b->batch && b->tokens && (!b->page_table || !b->length || !b->q_start))
    return say(FS_EINVAL, "page_table / length / q_start is NULL");
  return FS_OK;
}

int check_rows(const fs_kv_rows& r, const char* name) {
  if (!r.data) return say(FS_EINVAL, "%s is NULL", name);
  if (!aligned(r.data, 16)) return say(FS_EINVAL, "%s is not 16-byte aligned", name);
  if (r.token_stride % 8 || r.head_stride % 8 || r.token_stride < 0 || r.head_stride < 0)
    return say(FS_EINVAL, "%s: strides must be multiples of 8 elements, >= 0", name);
  return FS_OK;
}

KvView view_of(const fs_kv_cache* c, const fs_kv_batch* b, int q_heads, void* ws) {
  KvView v{};
  v.pages = c->pages;
  v.heads = c->heads;
  v.log_page = log2_page(c->page_tokens);
  v.batch = b->batch;
  v.tokens = b->tokens;
  v.max_new = b->max_new;
  v.max_length = b->max_length;
  v.table_stride = b->table_stride;
  v.group = q_heads / c->heads;
  v.k_scale = c->k_scale;
  v.v_scale = c->v_scale;
  v.page_table = b->page_table;
  v.length = b->length;
  v.q_start = b->q_start;
  v.status = static_cast<uint32_t*>(ws);
  return v;
}

// ---------------------------------------------------------------- append

struct KvAppendArgs {
  KvView v;
  uint8_t *kc, *vc;
  long long page_stride, head_stride, token_stride;
  const void *k, *vals, *q;
  void* q_out;
  long long k_token, k_head, v_token, v_head, q_token, q_head, o_token, o_head;
  const float *cos, *sin;
  int rot, angle_rows, interleaved, q_heads;
};

template <typename T>
__device__ __forceinline__ void unpack4(float (&x)[4], uint2 w) {
  const float2 a = Elem<T>::two(w.x), b = Elem<T>::two(w.y);
  x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
}

// The angles of the four dimensions from d0 on at position `pos`: one a pair (interleaved:
// two of each), or one a dimension.
struct Angles {
  float4 c, s;
};
__device__ __forceinline__ Angles angles_of(const KvAppendArgs& a, int pos, int d0) {
  Angles r{};
  if (d0 >= a.rot) return r;
  const int half = a.rot >> 1;
  const float* ct = a.cos + (long long)pos * half;
  const float* st = a.sin + (long long)pos * half;
  if (a.interleaved) {
    const float2 c = *reinterpret_cast<const float2*>(ct + (d0 >> 1)), s = *reinterpret_cast<const float2*>(st + (d0 >> 1));
    r.c = make_float4(c.x, c.x, c.y, c.y), r.s = make_float4(s.x, s.x, s.y, s.y);
  } else {
    const int i0 = d0 < half ? d0 : d0 - half;
    r.c = *reinterpret_cast<const float4*>(ct + i0), r.s = *reinterpret_cast<const float4*>(st + i0);
  }
  return r;
}

// What the dimensions from dA and from dB on are paired with: each other where the whole row is
// rotated in halves, their neighbours where pairs are interleaved, else what the row holds half
// the rotated dimensions away.
template <typename T>
__device__ __forceinline__ void partners(float (&pa)[4], float (&pb)[4], const float (&xa)[4], const float (&xb)[4],
                                         const T* row, int dA, int dB, const KvAppendArgs& a, int dim) {
  if (a.interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) pa[i] = xa[i ^ 1], pb[i] = xb[i ^ 1];
  } else if (a.rot == dim) {
#pragma unroll
    for (int i = 0; i < 4; ++i) pa[i] = xb[i], pb[i] = xa[i];
  } else {
    const int half = a.rot >> 1;
    uint2 wa = make_uint2(0, 0), wb = wa;
    if (dA < a.rot) wa = *reinterpret_cast<const uint2*>(row + (dA < half ? dA + half : dA - half));
    if (dB < a.rot) wb = *reinterpret_cast<const uint2*>(row + (dB < half ? dB + half : dB - half));
    unpack4<T>(pa, wa);
    unpack4<T>(pb, wb);
  }
}

// x rotated: x c - p s for the first of a pair, x c + p s for the second.
__device__ __forceinline__ void turn4(float (&x)[4], const float (&p)[4], int d0, const Angles& an, const KvAppendArgs& a) {
  if (d0 >= a.rot) return;
  const float c[4] = {an.c.x, an.c.y, an.c.z, an.c.w}, s[4] = {an.s.x, an.s.y, an.s.z, an.s.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float m = __fmul_rn(x[i], c[i]), n = __fmul_rn(p[i], s[i]);
    const bool first = a.interleaved ? !(i & 1) : d0 < (a.rot >> 1);
    x[i] = first ? __fsub_rn(m, n) : __fadd_rn(m, n);
  }
}

// Both groups of four dimensions of a row, rotated.
template <typename T>
__device__ __forceinline__ void rotate8(float (&x)[4], float (&y)[4], const T* row, int dA, int dB, const KvAppendArgs& a,
                                        int pos, int dim) {
  if (!a.rot) return;
  float px[4], py[4];
  partners<T>(px, py, x, y, row, dA, dB, a, dim);
  turn4(x, px, dA, angles_of(a, pos, dA), a);
  turn4(y, py, dB, angles_of(a, pos, dB), a);
}

template <typename T>
__device__ __forceinline__ void load4(float (&x)[4], const T* p) {
  unpack4<T>(x, *reinterpret_cast<const uint2*>(p));
}

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// The least power of two s >= 2^-126 with amax <= 448 s; 0 for 0. amax finite.
__device__ __forceinline__ float scale_for(float amax) {
  if (!(amax > 0.f)) return 0.f;
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 127;  // subnormals: -127, and the bound below holds
  const int p = e - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);  // 448 = 1.75 * 2^8
  return exp2_int(max(p, -126));
}

// Four values as codes: x / scale (the scale's reciprocal is exact), infinities saturated (an
// infinity times 0 would be NaN; the conversion saturates), NaN as 0.
__device__ __forceinline__ uint32_t codes4(const float (&x)[4], float inv) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = x[i] != x[i] ? 0.f : fabsf(x[i]) < INFINITY ? __fmul_rn(x[i], inv) : x[i];
  return e4m3x2(y[0], y[1]) | e4m3x2(y[2], y[3]) << 16;
}

// Eight codes under a scale that has grown: times f = old scale / new one.
__device__ __forceinline__ void rescale8(uint8_t* at, float f) {
  uint2* w = reinterpret_cast<uint2*>(at);
  const uint2 c = *w;
  uint32_t r[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t u = i ? c.y : c.x;
    const float2 lo = Elem<__half>::two(e4m3x2_to_f16x2(u)), hi = Elem<__half>::two(e4m3x2_to_f16x2_hi(u));
    r[i] = e4m3x2(__fmul_rn(lo.x, f), __fmul_rn(lo.y, f)) | e4m3x2(__fmul_rn(hi.x, f), __fmul_rn(hi.y, f)) << 16;
  }
  *w = make_uint2(r[0], r[1]);
}

// One unit of D / 8 lanes appends the new tokens of one (sequence, page) for one head
// of keys or values, or rotates one query head over them. Its lanes hold dimensions
// 4 l .. 4 l + 3 of each half. Two passes over the tokens: the largest magnitude,
// then the codes. For two to kFewTokens new tokens a sequence: latency (a chain of four
// loads: the sequence, its page, the page's scale, and the rows beside them).
template <int D, typename T>
__global__ void __launch_bounds__(128, 6) k_kv_append(const KvAppendArgs a) {
  constexpr int kLanes = D / 8, kUnits = 128 / kLanes;
  const int b = blockIdx.z, piece = blockIdx.x;
  const int unit = threadIdx.x / kLanes, l = threadIdx.x % kLanes;
  const int job = blockIdx.y * kUnits + unit;  // [0, heads) keys, [heads, 2 heads) values, then queries
  pdl_trigger();
  pdl_wait();
  KvSeq s;
  if (!kv_seq(a.v, b, s)) {
    if (threadIdx.x == 0) kv_flag(a.v, KV_ST_BATCH);
    return;
  }
  if (threadIdx.x == 0) kv_ends(a.v, b, s);
  const int P = 1 << a.v.log_page;
  const int p0 = max(s.len - s.count, 0);  // first position that is appended
  const int pg = (p0 >> a.v.log_page) + piece;
  const int lo = max(p0, pg << a.v.log_page), hi = min(s.len, (pg + 1) << a.v.log_page);
  if (lo >= hi || s.count == 0) return;
  const int H = a.v.heads;
  if (job >= 2 * H + (a.q ? a.q_heads : 0)) return;
  const long long row0 = (long long)s.first - (s.len - s.count);  // + position: the token's row
  if (a.rot && hi > a.angle_rows) {
    if (l == 0) kv_flag(a.v, KV_ST_ANGLE);
    return;
  }
  const int dA = 4 * l, dB = D / 2 + 4 * l;
  const uint32_t mask = (kLanes == 16 ? 0xffffu : 0xffu) << (threadIdx.x % 32 / kLanes * kLanes);  // the unit's lanes

  // Tokens go by twos: their loads are under way before the first store.
  if (job >= 2 * H) {
    const int h = job - 2 * H;
    for (int p = lo; p < hi; p += 2) {
      const int n = min(2, hi - p);
      float x[2][4], y[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (i < n) {
          const T* row = static_cast<const T*>(a.q) + (row0 + p + i) * a.q_token + h * a.q_head;
          load4(x[i], row + dA);
          load4(y[i], row + dB);
          rotate8<T>(x[i], y[i], row, dA, dB, a, p + i, D);
        }
      __syncwarp(mask);  // q_out may be q: every lane of a row has read before one writes
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (i < n) {
          T* to = static_cast<T*>(a.q_out) + (row0 + p + i) * a.o_token + h * a.o_head;
          *reinterpret_cast<uint2*>(to + dA) = make_uint2(Elem<T>::pack(x[i][0], x[i][1]), Elem<T>::pack(x[i][2], x[i][3]));
          *reinterpret_cast<uint2*>(to + dB) = make_uint2(Elem<T>::pack(y[i][0], y[i][1]), Elem<T>::pack(y[i][2], y[i][3]));
        }
    }
    return;
  }

  const bool is_k = job < H;
  const int h = is_k ? job : job - H;
  const T* src = is_k ? static_cast<const T*>(a.k) + row0 * a.k_token + h * a.k_head
                      : static_cast<const T*>(a.vals) + row0 * a.v_token + h * a.v_head;
  const long long src_token = is_k ? a.k_token : a.v_token;
  const int g = kv_page_raw(a.v, b, pg);
  if (!kv_page_held(a.v, g)) return;  // (all lanes of the unit)
  uint8_t* page = (is_k ? a.kc : a.vc) + g * a.page_stride + h * a.head_stride;
  float* scale_at = const_cast<float*>(is_k ? a.v.k_scale : a.v.v_scale) + (long long)g * H + h;
  const int slot0 = lo & (P - 1);
  const float old = slot0 ? *scale_at : 0.f;

  float amax = 0.f;
  bool nan = false;
#pragma unroll 2
  for (int p = lo; p < hi; ++p) {
    const T* row = src + p * src_token;
    float x[4], y[4];
    load4(x, row + dA);
    load4(y, row + dB);
    if (is_k) rotate8<T>(x, y, row, dA, dB, a, p, D);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float u = fabsf(x[i]), w = fabsf(y[i]);
      if (u < INFINITY) amax = fmaxf(amax, u);
      if (w < INFINITY) amax = fmaxf(amax, w);
      nan |= u != u || w != w;
    }
  }
  if (nan) kv_flag(a.v, KV_ST_VALUE);
#pragma unroll
  for (int o = kLanes / 2; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(mask, amax, o));
  const float now = fmaxf(old, scale_for(amax));
  if (slot0 && now > old) {
    // the page's earlier tokens, 8 codes a lane
    const float f = __fdiv_rn(old, now);
#pragma unroll 4
    for (int t = 0; t < slot0; ++t) rescale8(page + t * a.token_stride + 8 * l, f);
  }
  if (l == 0) *scale_at = now;

  const float inv = now > 0.f ? __fdiv_rn(1.f, now) : 0.f;
  for (int p = lo; p < hi; p += 2) {
    const int n = min(2, hi - p);
    float x[2][4], y[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (i < n) {
        const T* row = src + (p + i) * src_token;
        float u[4], w[4];
        load4(u, row + dA);
        load4(w, row + dB);
        if (is_k) rotate8<T>(u, w, row, dA, dB, a, p + i, D);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i][j] = u[j], y[i][j] = w[j];
      }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (i < n) {
        uint8_t* to = page + (long long)((p + i) & (P - 1)) * a.token_stride;
        *reinterpret_cast<uint32_t*>(to + dA) = codes4(x[i], inv);
        *reinterpret_cast<uint32_t*>(to + dB) = codes4(y[i], inv);
      }
  }
}

// The same for one new token a sequence at most: every load that does not need another's
// answer is under way at once, and few registers leave room for many units (256 sequences of
// 8 + 64 heads: 8 us on the GPU, 14 with the kernel above; 9 MB, so latency and not bandwidth).
template <int D, typename T>
__global__ void __launch_bounds__(128, 8) k_kv_append_one(const KvAppendArgs a) {
  constexpr int kLanes = D / 8, kUnits = 128 / kLanes;
  const int b = blockIdx.y, unit = threadIdx.x / kLanes, l = threadIdx.x % kLanes;
  const int job = blockIdx.x * kUnits + unit, H = a.v.heads;
  pdl_trigger();
  pdl_wait();
  KvSeq s;
  if (!kv_seq(a.v, b, s)) {
    if (threadIdx.x == 0) kv_flag(a.v, KV_ST_BATCH);
    return;
  }
  if (threadIdx.x == 0) kv_ends(a.v, b, s);
  const int p = s.len - 1;
  if (s.count == 0 || p < 0 || job >= 2 * H + (a.q ? a.q_heads : 0)) return;
  if (a.rot && p >= a.angle_rows) {
    if (l == 0) kv_flag(a.v, KV_ST_ANGLE);
    return;
  }
  const int dA = 4 * l, dB = D / 2 + 4 * l;
  const uint32_t mask = (kLanes == 16 ? 0xffffu : 0xffu) << (threadIdx.x % 32 / kLanes * kLanes);  // the unit's lanes
  const bool is_q = job >= 2 * H, is_k = job < H;
  const int h = is_q ? job - 2 * H : is_k ? job : job - H;
  const T* row = is_q   ? static_cast<const T*>(a.q) + s.first * a.q_token + h * a.q_head
                 : is_k ? static_cast<const T*>(a.k) + s.first * a.k_token + h * a.k_head
                        : static_cast<const T*>(a.vals) + s.first * a.v_token + h * a.v_head;
  const int g_raw = is_q ? 0 : kv_page_raw(a.v, b, p >> a.v.log_page);
  float x[4], y[4];
  load4(x, row + dA);
  load4(y, row + dB);
  if (is_q || is_k) rotate8<T>(x, y, row, dA, dB, a, p, D);
  if (is_q) {
    __syncwarp(mask);  // q_out may be q: every lane of a row has read before one writes
    T* to = static_cast<T*>(a.q_out) + s.first * a.o_token + h * a.o_head;
    *reinterpret_cast<uint2*>(to + dA) = make_uint2(Elem<T>::pack(x[0], x[1]), Elem<T>::pack(x[2], x[3]));
    *reinterpret_cast<uint2*>(to + dB) = make_uint2(Elem<T>::pack(y[0], y[1]), Elem<T>::pack(y[2], y[3]));
    return;
  }
  const int g = g_raw, slot = p & ((1 << a.v.log_page) - 1);
  if (!kv_page_held(a.v, g)) return;  // (all lanes of the unit)
  float* scale_at = const_cast<float*>(is_k ? a.v.k_scale : a.v.v_scale) + (long long)g * H + h;
  const float old = slot ? *scale_at : 0.f;
  float amax = 0.f;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float u = fabsf(x[i]), w = fabsf(y[i]);
    if (u < INFINITY) amax = fmaxf(amax, u);
    if (w < INFINITY) amax = fmaxf(amax, w);
    nan |= u != u || w != w;
  }
  if (nan) kv_flag(a.v, KV_ST_VALUE);
#pragma unroll
  for (int o = kLanes / 2; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(mask, amax, o));
  const float now = fmaxf(old, scale_for(amax));
  uint8_t* page = (is_k ? a.kc : a.vc) + g * a.page_stride + h * a.head_stride;
  if (slot && now > old) {
    const float f = __fdiv_rn(old, now);
#pragma unroll 4
    for (int t = 0; t < slot; ++t) rescale8(page + t * a.token_stride + 8 * l, f);
  }
  if (l == 0) *scale_at = now;
  const float inv = now > 0.f ? __fdiv_rn(1.f, now) : 0.f;
  uint8_t* to = page + slot * a.token_stride;
  *reinterpret_cast<uint32_t*>(to + dA) = codes4(x, inv);
  *reinterpret_cast<uint32_t*>(to + dB) = codes4(y, inv);
}

// The same for many new tokens: a block per (page, head of keys or values) holds the page's
// tokens in registers, kIt of them a unit, so that they are read once and all at once; for
// queries a block per page's tokens and kQHeads heads, whose rows share the angles. A unit a
// page, as above, keeps too few loads under way: 8 prompts of 4096 tokens took 389 us with it,
// 114 us with this one (623 MB, 5.5 TB/s, 80 % of the copy rate; issue slots 60 % busy).
constexpr int kQHeads = 8;
// Up to so many new tokens a sequence, k_kv_append. Measured on the GPU against k_kv_append_many (us, pages of 64
// tokens): it is the faster one for many sequences of many heads (8 + 64 heads, 256 sequences of 2, 4, 8, 9 tokens: 11, 17,
// 31, 37 against 30, 31, 35, 40; 64 of 2 and 4: 5.1 and 7.8 against 9.9 and 10.2, but 13.1 against 10.7 with 8), and the
// slower one elsewhere (one sequence of 2, 4, 8: 4.0, 6.1, 10.6 against 3.6, 3.7, 3.8; 1 + 8 heads, 64 sequences of 8: 11.1
// against 4.7; 64 sequences with pages of 16 of 8: 12.2 against 4.7). The rule does not look at sequences and heads.
constexpr int kFewTokens = 8;

template <int D, typename T, int kIt, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) k_kv_append_many(const KvAppendArgs a) {
  constexpr int kLanes = D / 8, kUnits = kThreads / kLanes;
  __shared__ float sm_amax[kThreads / 32];
  const int b = blockIdx.z, piece = blockIdx.x;
  const int unit = threadIdx.x / kLanes, l = threadIdx.x % kLanes;
  pdl_trigger();
  pdl_wait();
  KvSeq s;
  if (!kv_seq(a.v, b, s)) {
    if (threadIdx.x == 0) kv_flag(a.v, KV_ST_BATCH);
    return;
  }
  if (threadIdx.x == 0) kv_ends(a.v, b, s);
  const int P = 1 << a.v.log_page, H = a.v.heads;
  const int p0 = max(s.len - s.count, 0);
  const int pg = (p0 >> a.v.log_page) + piece;
  const int lo = max(p0, pg << a.v.log_page), hi = min(s.len, (pg + 1) << a.v.log_page);
  if (lo >= hi || s.count == 0) return;
  const long long row0 = (long long)s.first - (s.len - s.count);
  if (a.rot && hi > a.angle_rows) {
    if (threadIdx.x == 0) kv_flag(a.v, KV_ST_ANGLE);
    return;
  }
  const int dA = 4 * l, dB = D / 2 + 4 * l;

  if ((int)blockIdx.y >= 2 * H) {
    const int h0 = (blockIdx.y - 2 * H) * kQHeads, h_n = min(kQHeads, a.q_heads - h0);
    const uint32_t mask = (kLanes == 16 ? 0xffffu : 0xffu) << (threadIdx.x % 32 / kLanes * kLanes);
    if (a.rot == D && !a.interleaved) {
      // whole rows in halves: a lane holds eight dimensions and the eight they are paired with
      constexpr int kRowLanes = D / 16;
      const int ql = threadIdx.x % kRowLanes, d0 = 8 * ql;
      const uint32_t row_mask = ((1u << kRowLanes) - 1) << (threadIdx.x % 32 / kRowLanes * kRowLanes);
      for (int p = lo + threadIdx.x / kRowLanes; p < hi; p += kThreads / kRowLanes) {
        const T* from = static_cast<const T*>(a.q) + (row0 + p) * a.q_token + h0 * a.q_head + d0;
        T* to = static_cast<T*>(a.q_out) + (row0 + p) * a.o_token + h0 * a.o_head + d0;
        const float4* ct = reinterpret_cast<const float4*>(a.cos + (long long)p * (D / 2) + d0);
        const float4* st = reinterpret_cast<const float4*>(a.sin + (long long)p * (D / 2) + d0);
        const float4 c0 = ct[0], c1 = ct[1], s0 = st[0], s1 = st[1];
        const float c[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w}, sn[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll 1
        for (int hg = 0; hg < h_n; hg += 2, from += 2 * a.q_head, to += 2 * a.o_head) {  // two heads under way at a time
          uint4 x[2], y[2];
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (hg + h < h_n) {
              x[h] = *reinterpret_cast<const uint4*>(from + h * a.q_head);
              y[h] = *reinterpret_cast<const uint4*>(from + h * a.q_head + D / 2);
            }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t u[4] = {x[h].x, x[h].y, x[h].z, x[h].w}, w[4] = {y[h].x, y[h].y, y[h].z, y[h].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 m = Elem<T>::two(u[i]), n = Elem<T>::two(w[i]);
              u[i] = Elem<T>::pack(__fsub_rn(__fmul_rn(m.x, c[2 * i]), __fmul_rn(n.x, sn[2 * i])),
                                   __fsub_rn(__fmul_rn(m.y, c[2 * i + 1]), __fmul_rn(n.y, sn[2 * i + 1])));
              w[i] = Elem<T>::pack(__fadd_rn(__fmul_rn(n.x, c[2 * i]), __fmul_rn(m.x, sn[2 * i])),
                                   __fadd_rn(__fmul_rn(n.y, c[2 * i + 1]), __fmul_rn(m.y, sn[2 * i + 1])));
            }
            x[h] = make_uint4(u[0], u[1], u[2], u[3]), y[h] = make_uint4(w[0], w[1], w[2], w[3]);
          }
          __syncwarp(row_mask);  // q_out may be q: every lane of a row has read before one writes
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (hg + h < h_n) {
              *reinterpret_cast<uint4*>(to + h * a.o_head) = x[h];
              *reinterpret_cast<uint4*>(to + h * a.o_head + D / 2) = y[h];
            }
        }
      }
      return;
    }
    const int half = a.rot >> 1;
    if (a.interleaved || !(half & 7)) {
      // 16 bytes a lane: dimensions 8 l on; what they are paired with is in the lane itself, or in the one
      // that holds the dimensions half the rotated ones away
      const int d0 = 8 * l;
      const bool turns = d0 < a.rot, first = d0 < half;
      const int other = !turns || a.interleaved ? l : first ? l + (half >> 3) : l - (half >> 3);
      const int src = (threadIdx.x % 32 / kLanes) * kLanes + other;
      for (int p = lo + unit; p < hi; p += kUnits) {
        const T* from = static_cast<const T*>(a.q) + (row0 + p) * a.q_token + h0 * a.q_head + d0;
        T* to = static_cast<T*>(a.q_out) + (row0 + p) * a.o_token + h0 * a.o_head + d0;
        float c[8], sn[8];  // of each dimension (of pairs, twice); the sine negative for the first of a pair
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = 1.f, sn[i] = 0.f;
        if (turns) {
          const long long at = (long long)p * half + (a.interleaved ? d0 >> 1 : first ? d0 : d0 - half);
          const float4 c0 = *reinterpret_cast<const float4*>(a.cos + at), s0 = *reinterpret_cast<const float4*>(a.sin + at);
          if (a.interleaved) {
            const float cs[4] = {c0.x, c0.y, c0.z, c0.w}, ss[4] = {s0.x, s0.y, s0.z, s0.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) c[2 * i] = c[2 * i + 1] = cs[i], sn[2 * i] = -ss[i], sn[2 * i + 1] = ss[i];
          } else {
            const float4 c1 = *reinterpret_cast<const float4*>(a.cos + at + 4), s1 = *reinterpret_cast<const float4*>(a.sin + at + 4);
            const float cs[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w}, ss[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = cs[i], sn[i] = first ? -ss[i] : ss[i];
          }
        }
#pragma unroll 1
        for (int hg = 0; hg < h_n; hg += 4, from += 4 * a.q_head, to += 4 * a.o_head) {  // four heads under way at a time
          uint4 x[4];
#pragma unroll
          for (int h = 0; h < 4; ++h)
            if (hg + h < h_n) x[h] = *reinterpret_cast<const uint4*>(from + h * a.q_head);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          if (hg + h >= h_n) break;
          const uint32_t w[4] = {x[h].x, x[h].y, x[h].z, x[h].w};
          uint32_t y[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 u = Elem<T>::two(w[i]);
            const uint32_t pw = a.interleaved ? w[i] : __shfl_sync(mask, w[i], src);
            const float2 z = Elem<T>::two(pw);
            const float q0 = a.interleaved ? z.y : z.x, q1 = a.interleaved ? z.x : z.y;
            // (x c + p (-s) rounds as x c - p s does)
            const float r0 = __fadd_rn(__fmul_rn(u.x, c[2 * i]), __fmul_rn(q0, sn[2 * i]));
            const float r1 = __fadd_rn(__fmul_rn(u.y, c[2 * i + 1]), __fmul_rn(q1, sn[2 * i + 1]));
            y[i] = turns ? Elem<T>::pack(r0, r1) : w[i];
          }
          x[h] = make_uint4(y[0], y[1], y[2], y[3]);
        }
        __syncwarp(mask);  // q_out may be q: every lane of a row has read before one writes
#pragma unroll
        for (int h = 0; h < 4; ++h)
          if (hg + h < h_n) *reinterpret_cast<uint4*>(to + h * a.o_head) = x[h];
        }
      }
      return;
    }
    for (int p = lo + unit; p < hi; p += kUnits) {
      const Angles an = angles_of(a, p, dA), bn = angles_of(a, p, dB);
#pragma unroll 1
      for (int hg = 0; hg < h_n; hg += 4) {  // four heads' loads under way at a time
        const T* from = static_cast<const T*>(a.q) + (row0 + p) * a.q_token + (h0 + hg) * a.q_head;
        T* to = static_cast<T*>(a.q_out) + (row0 + p) * a.o_token + (h0 + hg) * a.o_head;
        uint2 x[4], y[4];
#pragma unroll
        for (int h = 0; h < 4; ++h)
          if (hg + h < h_n) {
            x[h] = *reinterpret_cast<const uint2*>(from + h * a.q_head + dA);
            y[h] = *reinterpret_cast<const uint2*>(from + h * a.q_head + dB);
          }
        if (a.rot) {
#pragma unroll
          for (int h = 0; h < 4; ++h)
            if (hg + h < h_n) {
              float u[4], w[4], pu[4], pw[4];
              unpack4<T>(u, x[h]);
              unpack4<T>(w, y[h]);
              partners<T>(pu, pw, u, w, from + h * a.q_head, dA, dB, a, D);
              turn4(u, pu, dA, an, a);
              turn4(w, pw, dB, bn, a);
              x[h] = make_uint2(Elem<T>::pack(u[0], u[1]), Elem<T>::pack(u[2], u[3]));
              y[h] = make_uint2(Elem<T>::pack(w[0], w[1]), Elem<T>::pack(w[2], w[3]));
            }
        }
        __syncwarp(mask);  // q_out may be q: every lane of a row has read before one writes
#pragma unroll
        for (int h = 0; h < 4; ++h)
          if (hg + h < h_n) {
            *reinterpret_cast<uint2*>(to + h * a.o_head + dA) = x[h];
            *reinterpret_cast<uint2*>(to + h * a.o_head + dB) = y[h];
          }
      }
    }
    return;
  }

  const bool is_k = (int)blockIdx.y < H;
  const int h = is_k ? blockIdx.y : blockIdx.y - H;
  const T* src = is_k ? static_cast<const T*>(a.k) + row0 * a.k_token + h * a.k_head
                      : static_cast<const T*>(a.vals) + row0 * a.v_token + h * a.v_head;
  const long long src_token = is_k ? a.k_token : a.v_token;
  const int g_raw = kv_page_raw(a.v, b, pg);
  float x[kIt][4], y[kIt][4];
  {
    uint2 xr[kIt], yr[kIt];
#pragma unroll
    for (int i = 0; i < kIt; ++i) {
      const int p = lo + unit + i * kUnits;
      xr[i] = yr[i] = make_uint2(0, 0);
      if (p < hi) {
        xr[i] = *reinterpret_cast<const uint2*>(src + p * src_token + dA);
        yr[i] = *reinterpret_cast<const uint2*>(src + p * src_token + dB);
      }
    }
#pragma unroll
    for (int i = 0; i < kIt; ++i) unpack4<T>(x[i], xr[i]), unpack4<T>(y[i], yr[i]);
  }
  if (is_k && a.rot) {
#pragma unroll
    for (int i = 0; i < kIt; ++i) {
      const int p = lo + unit + i * kUnits;
      if (p < hi) {
        float pu[4], pw[4];
        partners<T>(pu, pw, x[i], y[i], src + p * src_token, dA, dB, a, D);
        turn4(x[i], pu, dA, angles_of(a, p, dA), a);
        turn4(y[i], pw, dB, angles_of(a, p, dB), a);
      }
    }
  }
  float amax = 0.f;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < kIt; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float u = fabsf(x[i][j]), w = fabsf(y[i][j]);
      if (u < INFINITY) amax = fmaxf(amax, u);
      if (w < INFINITY) amax = fmaxf(amax, w);
      nan |= u != u || w != w;
    }
  if (nan) kv_flag(a.v, KV_ST_VALUE);
#pragma unroll
  for (int o = 16; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, o));
  if (threadIdx.x % 32 == 0) sm_amax[threadIdx.x / 32] = amax;
  const int g = g_raw;
  if (!kv_page_held(a.v, g)) return;  // (the whole block)
  float* scale_at = const_cast<float*>(is_k ? a.v.k_scale : a.v.v_scale) + (long long)g * H + h;
  const int slot0 = lo & (P - 1);
  const float old = slot0 ? *scale_at : 0.f;
  __syncthreads();  // (every thread has the old scale, too)
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) amax = fmaxf(amax, sm_amax[i]);
  const float now = fmaxf(old, scale_for(amax));
  uint8_t* page = (is_k ? a.kc : a.vc) + g * a.page_stride + h * a.head_stride;
  if (slot0 && now > old) {
    const float f = __fdiv_rn(old, now);
    for (int t = unit; t < slot0; t += kUnits) rescale8(page + t * a.token_stride + 8 * l, f);
  }
  if (threadIdx.x == 0) *scale_at = now;
  const float inv = now > 0.f ? __fdiv_rn(1.f, now) : 0.f;
#pragma unroll
  for (int i = 0; i < kIt; ++i) {
    const int p = lo + unit + i * kUnits;
    if (p < hi) {
      uint8_t* to = page + (long long)(p & (P - 1)) * a.token_stride;
      *reinterpret_cast<uint32_t*>(to + dA) = codes4(x[i], inv);
      *reinterpret_cast<uint32_t*>(to + dB) = codes4(y[i], inv);
    }
  }
}

template <int D, typename T>
cudaError_t launch_append(const KvAppendArgs& a, int pieces, bool many, cudaStream_t s) {
  const int q_heads = a.q ? a.q_heads : 0;
  constexpr int kUnits = 128 / (D / 8);
  const int unit_blocks = (2 * a.v.heads + q_heads + kUnits - 1) / kUnits;
  if (a.v.max_new == 1) return launch_pdl(k_kv_append_one<D, T>, dim3(unit_blocks, a.v.batch), dim3(128), 0, s, a);
  if (!many) return launch_pdl(k_kv_append<D, T>, dim3(pieces, unit_blocks, a.v.batch), dim3(128), 0, s, a);
  const dim3 grid(pieces, 2 * a.v.heads + (q_heads + kQHeads - 1) / kQHeads, a.v.batch);
  const int its = (D / 8 << a.v.log_page) / 128;  // rows a unit of a block of 128
  if (its <= 2) return launch_pdl(k_kv_append_many<D, T, 2, 128>, grid, dim3(128), 0, s, a);
  if (its == 4) return launch_pdl(k_kv_append_many<D, T, 4, 128>, grid, dim3(128), 0, s, a);
  if (its == 8) return launch_pdl(k_kv_append_many<D, T, 4, 256>, grid, dim3(256), 0, s, a);
  return launch_pdl(k_kv_append_many<D, T, 4, 512>, grid, dim3(512), 0, s, a);
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's encoder, looked up once (the library does not link libcuda).
EncodeTiled encode_tiled() {
  static const EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
        r != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return f;
}

int sm_count_of(int dev) {
  static std::atomic<int> known[64];
  if (dev < 0 || dev >= 64) return 0;
  int n = known[dev].load(std::memory_order_relaxed);
  if (!n && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess)
    known[dev].store(n, std::memory_order_relaxed);
  return n;
}

// How an attend call is cut up (see k_kv_decode): rows of a (sequence, key head) in tiles
// of row_tile, the cache axis in parts of `split` tokens.
struct KvPlan {
  int row_tile, row_blocks, split, splits, cluster, tickets;
  int chunk_tiles;  // blocks of k_kv_chunk a (sequence, key head); 0: no sequence has that many rows
  int chunk_split, chunk_parts;
  int few;          // sequences with more rows than this go to k_kv_chunk
  int wide_tiles;   // tiles of a sequence that k_kv_expand writes; 0: the walks convert for themselves
  int decode;       // whether some sequence can have few rows
  size_t part_floats, chunk_floats, wide_bytes;
};

// Sequences with more rows (new tokens x query heads of a key head) than kFewRows go to k_kv_chunk.
// With heads of 128, where k_kv_decode needs three passes over the codes (more than kMidRows) and
// k_kv_chunk's blocks fill at least half of the SMs, they go there too (us on the GPU, k_kv_decode against
// k_kv_chunk): 40 rows over 5 sequences of up to 40000 tokens 43 against 36, 64 rows over 48 of up to 6000 80
// against 61, 48 rows of 16 under a window of 4096 36 against 21, 40 rows 35 against 21; with one long sequence (16
// blocks) 24 against 33. With 32 rows: 48 sequences of up to 6000 46 against 60, but 16 under the window 30 against
// 21. Heads of 64 stay with k_kv_decode, though 40 rows over those 5 sequences take it 43 and k_kv_chunk 28.
constexpr int kMidRows = 32, kFewRows = 64;

// Where at least kWideFrom blocks can walk over a sequence's tokens, and the batch's tokens as
// halves take no more than kWideBytes, they are converted once. Measured, 16 sequences of 8 key heads (us, each walk
// converting against once): 2 blocks over 2000 tokens 80 against 107, 3 blocks 120 against 138, 4 blocks 156 against
// 166, 6 blocks 230 against 226, 8 blocks 269 against 260; over the new tokens alone 4 blocks 49 against 47, 8 blocks
// 100 against 90; with heads of 64 over 8000 tokens 3 blocks 296 against 306, 4 blocks 393 against 384.
constexpr int kWideFrom = 4;
constexpr long long kWideBytes = 1ll << 30;
void wide_of(const fs_kv_cache* c, const fs_kv_batch* b, int tiles, int* wide_tiles, size_t* bytes) {
  const long long per = (std::max(1, b->max_length) + 127) / 128;
  const long long all = per * b->batch * c->heads * (2ll * 128 * c->dim * 2);
  const bool wide = tiles >= kWideFrom && all <= kWideBytes;
  *wide_tiles = wide ? (int)per : 0;
  *bytes = wide ? (size_t)all : 0;
}

constexpr int kMinSplit = 128, kMaxSplit = 4096;

KvPlan plan_of(const fs_kv_cache* c, const fs_kv_batch* b, int q_heads, int window, int sms) {
  KvPlan p{};
  const long long all = (long long)std::max(1, b->max_new) * (q_heads / c->heads);
  p.few = kFewRows;
  if (all > kMidRows) {
    // parts of at least four tiles of 128 tokens where whole walks leave half of the SMs without a block
    // (more parts for balance alone cost more than they give: ragged chunks 105 us whole, 220 us in twos)
    p.chunk_tiles = (int)((all + kKvChunkRows - 1) / kKvChunkRows);
    const long long blocks = std::max(1, b->batch) * (long long)c->heads * p.chunk_tiles;
    const int walk = (std::max(1, window ? (int)std::min<long long>(b->max_length, (long long)window + kKvChunkRows + 126) : b->max_length) + 127) / 128;
    const long long want = std::max(1ll, std::min({sms / blocks, (long long)walk / 4, (long long)kKvFan}));
    const int tiles = (int)((walk + want - 1) / want);
    p.chunk_split = tiles * 128;
    p.chunk_parts = (walk + tiles - 1) / tiles;
    // (and where most sequences have all of those rows, the others with them: no second kernel for a few
    // that have fewer, or none. Measured, 2 key heads, five proposals for a share of 16 sequences of up to 9000
    // tokens and one token for the rest: one kernel 28 us, two 51, at shares of tokens from 0.75 on; below, where this
    // takes two, it is 28 to 30 against 53 to 57)
    if (c->dim == 128 && 2 * blocks * p.chunk_parts >= sms)
      p.few = all <= kFewRows && 4ll * b->tokens >= 3ll * b->batch * b->max_new ? 0 : kMidRows;
    if (all <= p.few) p.chunk_tiles = 0;
  }
  if (p.chunk_tiles) {
    wide_of(c, b, p.chunk_tiles, &p.wide_tiles, &p.wide_bytes);
    if (p.chunk_parts > 1) p.wide_tiles = 0, p.wide_bytes = 0;
    p.chunk_floats = p.chunk_parts > 1 ? (size_t)b->batch * c->heads * p.chunk_tiles * p.chunk_parts * kKvChunkRows * (c->dim + 4) : 0;
  }
  const int rows = (int)std::min<long long>(all, std::max(1, p.few));
  // (every sequence has max_new new tokens: all have the same rows, and k_kv_chunk takes whatever a
  // batch that breaks this has)
  p.decode = !p.chunk_tiles || (p.few && (long long)b->batch * b->max_new != b->tokens);
  p.row_tile = rows <= 8 ? 8 : 16;
  p.row_blocks = (rows + p.row_tile - 1) / p.row_tile;
  const long long items = (long long)std::max(1, b->batch) * c->heads * p.row_blocks;
  // (a window's tiles may begin up to 31 tokens early)
  const int len = std::max(1, window ? (int)std::min<long long>(b->max_length, (long long)window + b->max_new + 30) : b->max_length);
  p.tickets = p.cluster = 1;
  if (items > kKvTickets) {
    p.split = (len + 127) / 128 * 128;
    p.splits = 1;
  } else {
    // a part for every block that is resident at once; parts for three such waves where they are
    // few an item, because sequences differ in length (append and attention, 64 of up to 8192 tokens: 59 us, with one
    // wave 63, two 66, four 61)
    const long long slots = (long long)sms * (c->dim == 128 ? 3 : 6);
    const long long want = 2 * items <= slots ? slots / items : (3 * slots + items - 1) / items;
    p.split = std::clamp((int)((len + want - 1) / want + 127) / 128 * 128, kMinSplit, kMaxSplit);
    p.splits = (len + p.split - 1) / p.split;
    // clusters where blocks are few, or of few items. Measured on the GPU, one key head, tokens an item (us, with
    // clusters against without): 1 item of 1000 5.3 against 7.2, of 16384 10.3 against 11.5, of 131072 17.5
    // against 18.3; 8 of 4000 10.3 against 12.4. Where each item has many parts, the need of free places side by side
    // costs more: 8 of 65536 39 against 32 (clusters all the same), 16 of 65536 66 against 52 and 33 of 16384 41 against 30
    // (none). Between the two the rule is coarse: 12 of 4000 10.7 against 12.5, 33 of 1000 7.4 against 9.2 (none)
    if (items * p.splits <= (items <= 8 ? slots : sms))
      while (p.cluster < kKvCluster && p.cluster < p.splits) p.cluster *= 2;
    p.splits = (p.splits + p.cluster - 1) / p.cluster * p.cluster;
    const int groups = (p.splits / p.cluster + kKvFan - 1) / kKvFan;
    if (groups > 1 && items * (1 + groups) <= kKvTickets) p.tickets = 1 + groups;
  }
  p.part_floats = p.decode && p.splits > 1 ? (size_t)items * p.splits * p.row_tile * (c->dim + 2) : 0;
  return p;
}

// At least plan_of's part_floats, and nondecreasing in the batch's sizes: items * splits
// is at most 18 sms + 9 items (with whole clusters) where the items alone set the parts' length, items *
// ceil(len / kMaxSplit) where that does.
size_t part_floats_bound(const fs_kv_cache* c, const fs_kv_batch* b, int q_heads, int sms) {
  const long long rows = std::min<long long>(kFewRows, (long long)std::max(1, b->max_new) * (q_heads / c->heads));
  const long long items = std::min<long long>(kKvTickets, (long long)std::max(1, b->batch) * c->heads * ((rows + 7) / 8));
  const long long len = std::max(1, b->max_length);
  const long long decode = std::max(18ll * sms + (1 + kKvCluster) * items, items * ((len + kMaxSplit - 1) / kMaxSplit)) * 16 * (c->dim + 2);
  // chunks: at most sms parts in all
  const long long all = (long long)std::max(1, b->max_new) * (q_heads / c->heads);
  const long long blocks = all > kMidRows ? std::max(1, b->batch) * (long long)c->heads * ((all + kKvChunkRows - 1) / kKvChunkRows) : 0;
  // the tokens as halves, where a batch can have them at all: a smaller one may where a larger one's are too many
  const bool wide = all > (kWideFrom - 1) * (long long)kKvChunkRows;
  const long long tokens = ((len + 127) / 128) * std::max(1, b->batch) * c->heads * (2ll * 128 * c->dim * 2);
  return (size_t)(decode + std::min((long long)sms, kKvFan * blocks) * kKvChunkRows * (c->dim + 4) +
                  (wide ? std::min(tokens, kWideBytes) / 4 + 32 : 0));
}

int device_sms(int* sms) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_say(e, "cudaGetDevice");
  *sms = sm_count_of(dev);
  return *sms ? FS_OK : say(FS_ECUDA, "device query failed");
}

int check_workspace(const void* ws, int64_t bytes, int64_t need) {
  if (!ws) return say(FS_EINVAL, "workspace is NULL");
  if (!aligned(ws, 256)) return say(FS_EINVAL, "workspace is not 256-byte aligned");
  if (bytes < need)
    return say(FS_EINVAL, "workspace of %lld bytes is less than the %lld this call needs", (long long)bytes,
               (long long)need);
  return FS_OK;
}

}  // namespace

int kv_tensor_map(CUtensorMap* m, const fs_kv_cache& c, const void* base, int rows, bool swizzled) {
  const EncodeTiled enc = encode_tiled();
  if (!enc) return say(FS_ECUDA, "the driver has no cuTensorMapEncodeTiled");
  const cuuint64_t dims[4] = {(cuuint64_t)c.dim, (cuuint64_t)c.page_tokens, (cuuint64_t)c.heads, (cuuint64_t)c.pages};
  const cuuint64_t strides[3] = {(cuuint64_t)c.token_stride, (cuuint64_t)c.head_stride, (cuuint64_t)c.page_stride};
  const cuuint32_t box[4] = {(cuuint32_t)c.dim, (cuuint32_t)rows, 1, 1}, step[4] = {1, 1, 1, 1};
  const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(base), dims, strides, box, step,
                         CU_TENSOR_MAP_INTERLEAVE_NONE,
                         !swizzled ? CU_TENSOR_MAP_SWIZZLE_NONE
                         : c.dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? FS_OK : say(FS_ECUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
}

}  // namespace fs

using namespace fs;

extern "C" int fs_kv_workspace_bytes(const fs_kv_cache* cache, const fs_kv_batch* batch, int32_t q_heads,
                                     int64_t* bytes) {
  if (!bytes) return say(FS_EINVAL, "bytes is NULL");
  if (int rc = check_cache(cache)) return rc;
  fs_kv_batch b{};
  if (!batch) return say(FS_EINVAL, "batch is NULL");
  b = *batch;
  b.page_table = b.length = b.q_start = reinterpret_cast<const int32_t*>(16);  // (sizes alone are looked at)
  if (int rc = check_batch(cache, &b, q_heads)) return rc;
  if (q_heads % cache->heads) return say(FS_EINVAL, "q_heads = %d is not a multiple of %d heads", q_heads, cache->heads);
  int sms = 0;
  if (int rc = device_sms(&sms)) return rc;
  *bytes = (int64_t)(kKvPartAt + 4 * part_floats_bound(cache, &b, q_heads, sms));
  return FS_OK;
}

extern "C" int fs_kv_append(const fs_kv_cache* cache, const fs_kv_batch* batch, const fs_kv_new* in, void* workspace,
                            int64_t workspace_bytes, void* cuda_stream) {
  if (int rc = check_cache(cache)) return rc;
  if (!in) return say(FS_EINVAL, "rows is NULL");
  const bool with_q = in->q.data || in->q_out.data;
  if (int rc = check_batch(cache, batch, with_q ? in->q_heads : 1)) return rc;
  if (in->dtype != FS_KV_BF16 && in->dtype != FS_KV_FP16) return say(FS_EINVAL, "dtype = %d is not FS_KV_BF16 or FS_KV_FP16", in->dtype);
  if (in->rot < 0 || in->rot % 8 || in->rot > cache->dim)
    return say(FS_EINVAL, "rot = %d must be a multiple of 8 in [0, %d]", in->rot, cache->dim);
  if (in->interleaved != 0 && in->interleaved != 1) return say(FS_EINVAL, "interleaved = %d is not 0 or 1", in->interleaved);
  if (int rc = check_workspace(workspace, workspace_bytes, kKvPartAt)) return rc;
  if (batch->batch == 0 || batch->tokens == 0 || batch->max_new == 0) return FS_OK;
  if (in->rot) {
    if (!in->cos || !in->sin) return say(FS_EINVAL, "cos / sin is NULL with rot = %d", in->rot);
    if (!aligned(in->cos, 16) || !aligned(in->sin, 16)) return say(FS_EINVAL, "cos / sin are not 16-byte aligned");
    if (in->angle_rows < 1) return say(FS_EINVAL, "angle_rows = %d < 1", in->angle_rows);
  }
  if (int rc = check_rows(in->k, "k")) return rc;
  if (int rc = check_rows(in->v, "v")) return rc;
  if (with_q) {
    if (int rc = check_rows(in->q, "q")) return rc;
    if (int rc = check_rows(in->q_out, "q_out")) return rc;
  }
  KvAppendArgs a{};
  a.v = view_of(cache, batch, cache->heads, workspace);
  a.kc = static_cast<uint8_t*>(cache->k);
  a.vc = static_cast<uint8_t*>(cache->v);
  a.page_stride = cache->page_stride;
  a.head_stride = cache->head_stride;
  a.token_stride = cache->token_stride;
  a.k = in->k.data, a.k_token = in->k.token_stride, a.k_head = in->k.head_stride;
  a.vals = in->v.data, a.v_token = in->v.token_stride, a.v_head = in->v.head_stride;
  a.q = with_q ? in->q.data : nullptr, a.q_token = in->q.token_stride, a.q_head = in->q.head_stride;
  a.q_out = in->q_out.data, a.o_token = in->q_out.token_stride, a.o_head = in->q_out.head_stride;
  a.cos = in->cos, a.sin = in->sin;
  a.rot = in->rot, a.angle_rows = in->angle_rows, a.interleaved = in->interleaved, a.q_heads = in->q_heads;
  const int P = cache->page_tokens;
  const int pieces = (batch->max_new + P - 2) / P + 1;  // pages that max_new tokens can touch
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const bool h = in->dtype == FS_KV_FP16;
  const bool many = batch->max_new > kFewTokens;
  const cudaError_t e = cache->dim == 128 ? (h ? launch_append<128, __half>(a, pieces, many, s) : launch_append<128, __nv_bfloat16>(a, pieces, many, s))
                                          : (h ? launch_append<64, __half>(a, pieces, many, s) : launch_append<64, __nv_bfloat16>(a, pieces, many, s));
  return e == cudaSuccess ? FS_OK : cuda_say(e, "launch (fs_kv_append)");
}

extern "C" int fs_kv_attend(const fs_kv_cache* cache, const fs_kv_batch* batch, const fs_kv_query* qu, void* workspace,
                            int64_t workspace_bytes, void* cuda_stream) {
  if (int rc = check_cache(cache)) return rc;
  if (!qu) return say(FS_EINVAL, "query is NULL");
  if (int rc = check_batch(cache, batch, qu->q_heads)) return rc;
  if (qu->q_heads % cache->heads) return say(FS_EINVAL, "q_heads = %d is not a multiple of %d heads", qu->q_heads, cache->heads);
  if (qu->dtype != FS_KV_BF16 && qu->dtype != FS_KV_FP16) return say(FS_EINVAL, "dtype = %d is not FS_KV_BF16 or FS_KV_FP16", qu->dtype);
  if (!(std::fabs(qu->scale) < INFINITY)) return say(FS_EINVAL, "scale is not finite");
  if (qu->window < 0) return say(FS_EINVAL, "window = %d < 0", qu->window);
  if (batch->batch == 0 || batch->tokens == 0 || batch->max_new == 0) return check_workspace(workspace, workspace_bytes, kKvPartAt);
  if (int rc = check_rows(qu->q, "q")) return rc;
  if (int rc = check_rows(qu->out, "out")) return rc;
  int sms = 0;
  if (int rc = device_sms(&sms)) return rc;
  const int window = qu->window < batch->max_length ? qu->window : 0;  // (a window over everything is none)
  const KvPlan p = plan_of(cache, batch, qu->q_heads, window, sms);
  if (int rc = check_workspace(workspace, workspace_bytes, (int64_t)(kKvPartAt + 4 * (p.part_floats + p.chunk_floats) + (p.wide_bytes ? p.wide_bytes + 128 : 0)))) return rc;
  if (p.chunk_tiles > 65535) return say(FS_EINVAL, "max_new = %d: too many rows for one call", batch->max_new);

  KvAttendArgs a{};
  a.v = view_of(cache, batch, qu->q_heads, workspace);
  a.q = qu->q.data, a.q_token = qu->q.token_stride, a.q_head = qu->q.head_stride;
  a.out = qu->out.data, a.out_token = qu->out.token_stride, a.out_head = qu->out.head_stride;
  a.scale_log2 = qu->scale * 1.44269504f;
  a.window = window;
  a.split = p.split;
  a.tickets = p.tickets;
  a.cluster = p.cluster;
  a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + kKvPartAt);
  a.ticket = reinterpret_cast<unsigned*>(static_cast<char*>(workspace) + kKvTicketAt);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  CUtensorMap mk, mv;
  if (p.chunk_tiles) {
    KvAttendArgs ca = a;
    ca.min_rows = p.decode ? p.few : 0, ca.max_rows = batch->max_new * (qu->q_heads / cache->heads);
    ca.split = p.chunk_split;
    ca.part = a.part + p.part_floats;
    ca.wide_tiles = p.wide_tiles;
    if (p.wide_tiles)
      ca.wide = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(ca.part + p.chunk_floats) + 127) & ~(uintptr_t)127);
    if (int rc = kv_tensor_map(&mk, *cache, cache->k, cache->page_tokens, false)) return rc;
    if (int rc = kv_tensor_map(&mv, *cache, cache->v, cache->page_tokens, false)) return rc;
    const cudaError_t e = launch_kv_chunk(mk, mv, ca, *cache, qu->dtype, p.chunk_tiles, p.chunk_parts, st);
    if (e != cudaSuccess) return cuda_say(e, "launch (fs_kv_attend, chunks)");
  }
  if (p.decode) {
    a.min_rows = 0, a.max_rows = p.few;
    const int box = std::min(32, cache->page_tokens);
    if (int rc = kv_tensor_map(&mk, *cache, cache->k, box, true)) return rc;
    if (int rc = kv_tensor_map(&mv, *cache, cache->v, box, true)) return rc;
    const cudaError_t e = launch_kv_decode(mk, mv, a, cache->dim, qu->dtype, p.row_tile, p.row_blocks, p.splits, st);
    if (e != cudaSuccess) return cuda_say(e, "launch (fs_kv_attend)");
  }
  return FS_OK;
}

extern "C" int fs_kv_check(void* workspace, void* cuda_stream) {
  if (int rc = check_workspace(workspace, kKvPartAt, kKvPartAt)) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  uint32_t st = 0;
  cudaError_t e = cudaMemcpyAsync(&st, workspace, 4, cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) return cuda_say(e, "synchronize (fs_kv_check)");
  if (!st) return FS_OK;
  e = cudaMemsetAsync(workspace, 0, kKvPartAt, s);  // a wait that ran out leaves tickets behind
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) return cuda_say(e, "clear (fs_kv_check)");
  if (st & ST_TIMEOUT) return say(FS_ETIMEOUT, "a device wait timed out (status 0x%x)", st);
  return say(FS_EDEVICE, "%s%s%s%s%s(status 0x%x)", st & KV_ST_PAGE ? "a page id outside the cache; " : "",
             st & KV_ST_BATCH ? "length or q_start out of the batch's bounds; " : "",
             st & KV_ST_VALUE ? "a NaN in keys or values; " : "",
             st & KV_ST_ANGLE ? "a position beyond the rows of cos / sin; " : "",
             st & KV_ST_SCALE ? "a scale that is neither a power of two nor 0, or scales of values of a sequence 2^100 apart; " : "", st);
}
