// Attention of many rows over the paged 8-bit cache (chunks of prompts): tcgen05.
//
// A block takes two tiles of 128 rows (new token, query head) of one (sequence, key head)
// and walks over the cache in tiles of 128 tokens:
//   S [128 x 128] = Q K^T,  P = 2^(c S + e - m),  O [128 x dim] += P V
// with both products on the tensor cores in half precision (the codes are exact in it, a
// bf16 query too once its row is scaled by a power of two; P keeps 11 bits) and S, P, O in
// tensor memory: S_t in 128 columns, P_t in the first 64 of the same ones (a row's thread
// holds its S in registers by then), O_t in dim. c holds the scale of a page's keys, e is log2
// of that of its values and m the largest of c S + e: half precision's step in P is relative to
// what counts most, however far the scales are apart. The row's sum of weights is taken in
// float without e. O is rescaled only when m has grown by more than 2^8 (P, times 2^7, stays
// under 65504), so almost never after the first tiles.
//
// The codes become halves once for all walks (k_kv_expand) where at least four blocks walk over
// a sequence's tokens, else in each walk. Roles of the warps:
//   0-3, 4-7  softmax of tile 0 / 1, a row a thread. Half of P is handed over while the other half
//             is computed (471 -> 465 us, see below). Two threads a row: 544 us, the 16 warps
//             crowd out the one that issues products
//   8-11      (only where the walk converts) codes to halves, from the tiles as they came to
//             swizzled ones; two warps for the keys, two for the values
//   then one  issues every product. While tile 0's rows are in softmax the tensor cores work on
//             tile 1, and the other way round. Two such warps, one a tile: 506-525 us, their
//             products mix and neither chain is short
//   and one   keeps tiles on their way: bulk copies of 32 KB halves, or tensor-map copies of the
//             codes, a page each at most: of the keys, and one more warp of the values (one for both
//             took 2900 clocks a tile beside the other warps, longer than anything else)
//
// Where the rows end in the first tile, the second's warps and tensor memory take every second tile of
// the cache for the same rows, and both results are joined at the end (with the warps for keys and values:
// 64 rows over 48 sequences of up to 6000 tokens 96 -> 78 us).
//
// Bound by the tensor cores, 4 dim operations per (row, token), and by how fast one thread beside
// eight busy softmax warps can issue their products and waits (a commit costs it about 200 clocks,
// so a slot is refilled after the S that follows its products and there are only the two of S a pair
// of tiles: 477 -> 458 us with three, 411 -> 407 with two). A prompt of 8192 tokens, 32 query heads over 4
// key heads of 128: 390 us with the conversion, 1.41 PFLOP/s of causal work, tensor cores active
// 64 % of the time; 73 % of the bf16 rate that a library product reaches. The steps in brackets are of the same prompt, when they were taken.
#include "fs_kv.cuh"
#include "fs_tc.cuh"

namespace fs {
namespace {

constexpr int kTok = 128, kTileRows = 128;
constexpr float kUp = 7.f;  // halves hold 2^(kUp + 8) of a row's largest weight

template <int D, bool kWide>
struct Cfg {
  static constexpr int kThreads = kWide ? 12 * 32 : 16 * 32;
  static constexpr int kIssuer = kWide ? 8 : 12;          // the warp that issues the products, and the next one that copies
  static constexpr int kStages = D == 128 ? 4 : 8;        // tiles of halves
  static constexpr int kRaw = kWide ? 0 : D == 128 ? 2 : 4;  // tiles of codes
  static constexpr int kSlot = kTok * D * 2, kRawSlot = kTok * D;
  static constexpr int kQ = 2 * kTileRows * D * 2;
  static constexpr size_t kSmem = 1024 + kQ + (size_t)kStages * kSlot + kRaw * kRawSlot + 1792;
};

// S of tile j of the cache is told on barrier j mod kRound. (Whoever refills a slot waits for the S
// after the products that read it, up to four tiles late: a barrier must not be two phases on by then.)
constexpr int kRound = 4;

struct Bars {
  uint64_t full[8], raw_full[4], raw_empty[4], s_full[2][kRound], p_full[2][2], pv_done[2], end;
  float vs[4][8];        // per tile of codes and 16 tokens: the values' scale
  uint32_t cut[4];       // per tile of codes: some tokens' values are to be 0
  float2 scale[16][8];   // per tile (mod 16) and 16 tokens: the keys' scale, log2 of the values' over the first page's
  float v_ref;
  uint32_t tmem;
};
static_assert(sizeof(Bars) <= 1792, "the barriers' share of shared memory");

__device__ __forceinline__ void st_shared16(uint32_t a, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

__device__ __forceinline__ uint4 ld_shared16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}

__device__ __forceinline__ float2 ld_shared8(uint32_t a) {
  float2 v;
  asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a) : "memory");
  return v;
}

// Two floats at a time (one instruction each).
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n .reg .b64 a, b, c, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n"
      " fma.rn.f32x2 d, a, b, c;\n mov.b64 {%0, %1}, d;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n add.rn.f32x2 d, a, b;\n mov.b64 {%0, %1}, d;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// half x half -> float products of 128 rows and n columns; b_mn: B's columns are contiguous
__host__ __device__ constexpr uint32_t instr_desc(int n, bool b_mn) {
  return 1u << 4 | (b_mn ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (uint32_t)(128 >> 4) << 24;
}

__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t a, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(a),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// Global -> shared copy of a contiguous tile.
__device__ __forceinline__ void bulk_g2s_at(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

// A wait that says so when it runs out; the caller leaves its loop.
__device__ __forceinline__ bool wait_bar(uint64_t* bar, uint32_t parity, const KvView& v) {
  if (mbar_wait(bar, parity, kWaitLimitNs)) return true;
  kv_flag(v, ST_TIMEOUT);
  return false;
}

// A row of S: its largest log2 weight (times its value scale) among columns [lo, hi] (all of
// them with kWhole); masked columns become -infinity.
template <bool kWhole>
__device__ __forceinline__ float row_top(float (&x)[kTok], float c, const float2* scale, int lo, int hi) {
  float top = -INFINITY;
#pragma unroll
  for (int g = 0; g < kTok / 16; ++g) {
    if (!kWhole) {
#pragma unroll
      for (int i = 16 * g; i < 16 * g + 16; ++i)
        if (i > hi || i < lo) x[i] = -INFINITY;
    }
    const float* y = x + 16 * g;
    const float m0 = max3(max3(max3(y[0], y[1], y[2]), max3(y[3], y[4], y[5]), max3(y[6], y[7], y[8])),
                          max3(y[9], y[10], y[11]), max3(max3(y[12], y[13], y[14]), y[15], y[15]));
    if (kWhole || m0 > -INFINITY) top = fmaxf(top, fmaf(m0, c * scale[g].x, scale[g].y));
  }
  return top;
}

// The keys that rows [r0, r_end) of a sequence see, from `first` on: a walk over [begin, end), in
// parts of a.split tokens.
struct Walk {
  int first, begin, end, parts;
};
__device__ __forceinline__ Walk walk_of(const KvAttendArgs& a, const KvSeq& s, int r0, int r_end) {
  const int base = s.len - s.count;
  const int pos0 = base + r0 / a.v.group, pos1 = base + (r_end - 1) / a.v.group;
  Walk w;
  w.end = max(pos1 + 1, 0);
  w.first = a.window ? max(pos0 - a.window + 1, 0) : 0;
  w.begin = w.first & ~(kTok - 1);
  w.parts = max(1, (w.end - w.begin + a.split - 1) / a.split);
  return w;
}

template <int D, typename T, bool kWide>
__global__ void __launch_bounds__(Cfg<D, kWide>::kThreads, 1) k_kv_chunk(const __grid_constant__ CUtensorMap mk,
                                                             const __grid_constant__ CUtensorMap mv, const KvAttendArgs a) {
  using C = Cfg<D, kWide>;
  constexpr int kPart = 2 * kTileRows * (D + 4);  // floats of a part's result: per row its sums, m, l (and two to keep 16 bytes)
  extern __shared__ unsigned char raw[];
  const uint32_t smem = (smem_u32(raw) + 1023) & ~1023u;
  const uint32_t q_at = smem, ring_at = smem + C::kQ, raw_at = ring_at + C::kStages * C::kSlot;
  Bars& bars = *reinterpret_cast<Bars*>(raw + (smem - smem_u32(raw)) + C::kQ + (size_t)C::kStages * C::kSlot +
                                        C::kRaw * C::kRawSlot);
  const KvView& v = a.v;
  const int h = blockIdx.x % v.heads, b = blockIdx.x / v.heads;
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int item = blockIdx.y * gridDim.x + blockIdx.x;

  pdl_trigger();
  pdl_wait();
  KvSeq s;
  if (!kv_seq(v, b, s)) {
    if (threadIdx.x == 0 && blockIdx.y == 0) kv_flag(v, KV_ST_BATCH);
    return;
  }
  if (threadIdx.x == 0 && blockIdx.y == 0) kv_ends(v, b, s);
  // each sequence's last rows first: theirs are its longest walks
  const int rows = s.count * v.group, part = blockIdx.z;
  const int tile = (rows + 2 * kTileRows - 1) / (2 * kTileRows) - 1 - (int)blockIdx.y, r0 = tile * (2 * kTileRows);
  if (tile < 0 || rows <= a.min_rows || rows > a.max_rows) return;
  const int r_end = min(rows, r0 + 2 * kTileRows);
  const int n_sub = r_end - r0 > kTileRows ? 2 : 1;
  const int base = s.len - s.count;  // position of the sequence's first new token
  const Walk walk = walk_of(a, s, r0, r_end);
  const int n_parts = walk.parts;
  if (n_parts > (int)gridDim.z) {  // a length beyond max_length
    if (threadIdx.x == 0 && part == 0) kv_flag(v, KV_ST_BATCH);
    return;
  }
  if (part >= n_parts) return;
  const int begin = walk.begin + part * a.split, kv_hi = min(begin + a.split, walk.end);  // this block's part
  const int n = (kv_hi - begin + kTok - 1) / kTok;  // tiles of the cache; 0: no row sees a token
  // With one tile of rows, each half of the block (softmax warps, S, O) takes every second tile of the
  // cache, and the halves' results are joined at the end.
  const bool two = !kWide && n_sub == 1 && n > 1;
  const int n_act = two ? 2 : n_sub;
  // (where the second tile's queries would be are then two more tiles of codes)
  const int n_raw = D == 128 && two ? 4 : C::kRaw;
  auto raw_slot = [&](int rs) { return rs < C::kRaw ? raw_at + rs * C::kRawSlot : q_at + kTileRows * D * 2 + (rs - C::kRaw) * C::kRawSlot; };

  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kStages; ++i) mbar_init(&bars.full[i], kWide ? 1 : 64);
    for (int i = 0; i < n_raw; ++i) mbar_init(&bars.raw_full[i], 1), mbar_init(&bars.raw_empty[i], 64);
    for (int t = 0; t < 2; ++t) {
      for (int i = 0; i < kRound; ++i) mbar_init(&bars.s_full[t][i], 1);
      mbar_init(&bars.p_full[t][0], 128), mbar_init(&bars.p_full[t][1], 128), mbar_init(&bars.pv_done[t], 1);
    }
    mbar_init(&bars.end, 1);
    bars.v_ref = 1.f;
  }
  if (w == C::kIssuer) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&bars.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  __syncthreads();

  // queries: a row a thread, scaled into [-2, 2] by a power of two (and by the scale's sign); every load
  // under way at once (8192-token prompt 402 -> 392 us)
  int q_exp = 0;
  if (w < 8) {
    const int r = r0 + (two ? threadIdx.x & 127 : threadIdx.x);
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + (long long)(s.first + r / v.group) * a.q_token +
                                                    (h * v.group + r % v.group) * a.q_head);
    uint4 u[D / 8];
#pragma unroll
    for (int i = 0; i < D / 8; ++i) u[i] = r < r_end ? q[i] : make_uint4(0, 0, 0, 0);
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      const float2 z0 = Elem<T>::two(u[i].x), z1 = Elem<T>::two(u[i].y), z2 = Elem<T>::two(u[i].z), z3 = Elem<T>::two(u[i].w);
      amax = fmaxf(amax, fmaxf(fmaxf(fmaxf(fabsf(z0.x), fabsf(z0.y)), fmaxf(fabsf(z1.x), fabsf(z1.y))),
                               fmaxf(fmaxf(fabsf(z2.x), fabsf(z2.y)), fmaxf(fabsf(z3.x), fabsf(z3.y)))));
    }
    q_exp = row_exponent(amax);
    const float down = a.scale_log2 < 0.f ? -exp2_int(-q_exp) : exp2_int(-q_exp);
    const int t = threadIdx.x >> 7, rr = threadIdx.x & 127;
    const uint32_t row = q_at + t * (kTileRows * D * 2) + rr * 128;
    if (!two || t == 0) {
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        uint32_t y[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 z = Elem<T>::two(y[k]);
          y[k] = pack_f16(z.x * down, z.y * down);
        }
        st_shared16(row + (i >> 3) * (kTileRows * 128) + (((i & 7) ^ (rr & 7)) << 4), make_uint4(y[0], y[1], y[2], y[3]));
      }
    }
    fence_proxy_async();
  }
  // Queries are in place: only the warps that stored them and the one that issues products wait for
  // that; tiles of the cache are on their way meanwhile.
  if (w < 8 || w == C::kIssuer) {
    fence_before();
    asm volatile("bar.sync 1, 288;" ::: "memory");
    fence_after();
  }
  // (the whole of tensor memory is this block's: its columns begin at 0)
  constexpr uint32_t tmem = 0;

  // Registers at launch: 512 threads x 128 (384 x 168); from here on 128 x (192 + 192 + 80 + 48)
  // (128 x (192 + 192 + 120)).
  if (w < 8) {
    // ---------------------------------------------------------------- softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
    const int t = w >> 2;
    const int r = r0 + (two ? threadIdx.x & 127 : threadIdx.x);
    if (t < n_act) {
      const uint32_t lanes = (uint32_t)(w & 3) << 21;  // 32 lanes a warp, in bits 16 and up
      const uint32_t s_at = tmem + lanes + t * 128, o_at = tmem + lanes + 256 + t * 128;
      const float c = fabsf(a.scale_log2) * exp2_int(q_exp);
      const int pos = base + r / v.group;
      const int hi = r < r_end ? pos : -1, lo = a.window ? pos - a.window + 1 : 0;
      // tiles inside [all_lo, all_hi) are seen whole by every row of this tile
      const int t_r0 = two ? r0 : r0 + t * kTileRows, t_r1 = min(r_end, t_r0 + kTileRows) - 1;
      const int all_hi = base + t_r0 / v.group + 1, all_lo = a.window ? base + t_r1 / v.group - a.window + 1 : 0;
      float m = -INFINITY, l = 0.f;
      bool ok = true;
      const int first = two ? t : 0, step = two ? 2 : 1;
      for (int j = first; j < n; j += step) {
        const int t0 = begin + j * kTok;
        const bool whole = t0 >= all_lo && t0 + kTok <= all_hi;
        const int c_hi = hi - t0, c_lo = lo - t0;  // columns [c_lo, c_hi] count
        ok = wait_bar(&bars.s_full[t][j % kRound], (j / kRound) & 1, v);
        if (!__all_sync(~0u, ok)) break;
        fence_after();
        float x[kTok];
#pragma unroll
        for (int k = 0; k < 4; ++k) tmem_ld32(reinterpret_cast<uint32_t(&)[32]>(x[32 * k]), s_at + 32 * k);
        wait_ld();
        const float2* scale = bars.scale[j & 15];
        const float top = whole ? row_top<true>(x, c, scale, 0, 0) : row_top<false>(x, c, scale, c_lo, c_hi);
        const bool grow = top > m + 8.f || (m == -INFINITY && top > m);
        if (__any_sync(~0u, grow)) {
          const float f = grow ? ex2(m - top) : 1.f;
          if (grow) m = top;
          l *= f;
          if (j > first) {  // (the first product overwrites O; those before this S have ended with it)
#pragma unroll 1
            for (int k = 0; k < D / 16; ++k) {
              uint32_t y[16];
              tmem_ld16(y, o_at + 16 * k);
              wait_ld();
#pragma unroll
              for (int i = 0; i < 16; ++i) y[i] = __float_as_uint(__uint_as_float(y[i]) * f);
              tmem_st16(o_at + 16 * k, y);
            }
          }
        }
        const float off = m == -INFINITY ? 0.f : m;  // (m: log2 of weight times scale, without kUp)
        // P = 2^(c S + log2 of the value scale - m), and the row's sum of weights without the scales
        // (a masked column: c times -infinity, but c may be 0)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t p[16];
#pragma unroll
          for (int g = 2 * k; g < 2 * k + 2; ++g) {
            const float ve = scale[g].y, off_g = ve + kUp - off;
            const float cg = whole ? c * scale[g].x : fmaxf(c * scale[g].x, 0x1p-126f);
            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 16 * g; i < 16 * g + 16; i += 2) {
              float2 y = fma2(make_float2(x[i], x[i + 1]), make_float2(cg, cg), make_float2(off_g, off_g));
              y.x = ex2(y.x), y.y = ex2(y.y);
              sum = add2(sum, y);
              p[(i - 32 * k) / 2] = pack_f16(y.x, y.y);
            }
            l = fmaf(sum.x + sum.y, exp2_int(-(int)ve - 7), l);
          }
          tmem_st16(s_at + 16 * k, p);
          if (k & 1) {  // half of P: its product begins while the other half is computed
            wait_st();
            fence_before();
            mbar_arrive(&bars.p_full[t][k >> 1]);
          }
        }
      }
      // ------------------------------------------------------------ result
      if (ok && n > 0) {
        ok = wait_bar(&bars.pv_done[t], 0, v);
        fence_after();
      }
      ok = __all_sync(~0u, ok);
      // the halves' results: the second's through shared memory (the tiles' slots, which nothing uses
      // once both halves' products have ended)
      float f0 = 1.f, f1 = 0.f;
      const uint32_t mine = ring_at + (threadIdx.x & 127) * ((D + 4) * 4);
      if (two) {
        asm volatile("bar.sync 2, 256;" ::: "memory");
        if (t == 1) {
#pragma unroll 1
          for (int k = 0; k < D / 16; ++k) {
            uint32_t x[16];
            tmem_ld16(x, o_at + 16 * k);
            wait_ld();
#pragma unroll
            for (int i = 0; i < 16; i += 4) st_shared16(mine + (16 * k + i) * 4, make_uint4(x[i], x[i + 1], x[i + 2], x[i + 3]));
          }
          st_shared16(mine + D * 4, make_uint4(__float_as_uint(m), __float_as_uint(l), ok, 0));
        }
        asm volatile("bar.sync 2, 256;" ::: "memory");
        if (t == 0) {
          const uint4 other = ld_shared16(mine + D * 4);
          const float m1 = __uint_as_float(other.x), top = fmaxf(m, m1), off = top == -INFINITY ? 0.f : top;
          f0 = ex2(m - off), f1 = ex2(m1 - off);
          m = top, l = fmaf(__uint_as_float(other.y), f1, l * f0);
          ok = __all_sync(~0u, ok && other.z);
        }
      }
      auto result = [&](uint32_t(&x)[32], int k) {
        tmem_ld32(x, o_at + 32 * k);
        wait_ld();
        if (two) {
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const uint4 y = ld_shared16(mine + (32 * k + i) * 4);
            const uint32_t ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int u = 0; u < 4; ++u) x[i + u] = __float_as_uint(fmaf(__uint_as_float(ys[u]), f1, __uint_as_float(x[i + u]) * f0));
          }
        }
      };
      const float up = bars.v_ref * (1.f / 128.f), inv = up / l;
      if (two && t == 1) {
        // (its result is the first half's)
      } else if (n_parts == 1) {
        T* to = static_cast<T*>(a.out) + (long long)(s.first + r / v.group) * a.out_token + (h * v.group + r % v.group) * a.out_head;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
          uint32_t x[32];
          if (n > 0) result(x, k);
          if (ok && r < r_end) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t y[4];
#pragma unroll
              for (int u = 0; u < 4; ++u)
                y[u] = l != 0.f ? Elem<T>::pack(__uint_as_float(x[8 * i + 2 * u]) * inv, __uint_as_float(x[8 * i + 2 * u + 1]) * inv) : 0u;
              *reinterpret_cast<uint4*>(to + 32 * k + 8 * i) = make_uint4(y[0], y[1], y[2], y[3]);
            }
          }
        }
      } else {
        float* to = a.part + ((long long)item * gridDim.z + part) * kPart + threadIdx.x * (D + 4);
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
          uint32_t x[32];
          result(x, k);
          if (r < r_end) {
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              *reinterpret_cast<float4*>(to + 32 * k + i) = make_float4(__uint_as_float(x[i]) * up, __uint_as_float(x[i + 1]) * up,
                                                                        __uint_as_float(x[i + 2]) * up, __uint_as_float(x[i + 3]) * up);
          }
        }
        if (r < r_end) *reinterpret_cast<float2*>(to + D) = make_float2(m, l);
      }
    }
  } else if (!kWide && w < 12) {
    // ---------------------------------------------------------------- codes to halves
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    // Two warps for the keys, two for the values: while one pair waits for its tile the other converts.
    constexpr int kLanes = D / 16;               // lanes a token, 16 codes each
    constexpr int kPer = 64 / kLanes;            // tokens a pass
    constexpr int kPasses = 8, kBatches = kTok / kPer / kPasses;  // (2 of 8 passes with dim 128)
    const bool values = w >= 10;
    const int id = threadIdx.x & 63, cl = id % kLanes, tk = id / kLanes;
    // A lane's 16 codes become the 16-byte chunks 2 (cl mod 4) and + 1 of the token's row in block
    // cl / 4; lanes of the second block begin with the other one, so that a row's lanes meet every
    // bank once.
    const int sw = D == 128 ? cl >> 2 : 0;
    const uint32_t from = tk * D + cl * 16, to = (cl >> 2) * (kTok * 128) + tk * 128;
    const uint32_t c0 = (((cl & 3) * 2 + sw) ^ (tk & 7)) << 4, c1 = (((cl & 3) * 2 + (sw ^ 1)) ^ (tk & 7)) << 4;
    int rs = values, st = values;
    uint32_t rs_par = 0;
    for (int j = 0; j < n; ++j) {
      bool ok = wait_bar(&bars.raw_full[rs], rs_par, v);
      if (!ok) break;
      const bool cut = values && bars.cut[rs];
      const uint32_t slot = raw_slot(rs) + from, row = ring_at + st * C::kSlot + to;
#pragma unroll
      for (int q = 0; q < kBatches; ++q) {
        uint32_t x[kPasses][4];
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
          const uint32_t at = slot + (q * kPasses + p) * (kPer * D);
          const float2 u = ld_shared8(at + 8 * sw), z = ld_shared8(at + 8 * (sw ^ 1));
          x[p][0] = __float_as_uint(u.x), x[p][1] = __float_as_uint(u.y);
          x[p][2] = __float_as_uint(z.x), x[p][3] = __float_as_uint(z.y);
        }
        if (cut) {
          // tokens that no row sees (their slots may hold NaN codes), and values whose scale is 0
#pragma unroll
          for (int p = 0; p < kPasses; ++p) {
            const int tl = (q * kPasses + p) * kPer + tk;
            if (begin + j * kTok + tl >= kv_hi || bars.vs[rs][tl >> 4] == 0.f) x[p][0] = x[p][1] = x[p][2] = x[p][3] = 0;
          }
        }
        if (q == kBatches - 1) mbar_arrive(&bars.raw_empty[rs]);
        // the slot's last tile, kStages / 2 of the cache's tiles ago (the last S of tile j follows the
        // products over its keys and over the values of the tile before: of its half, where the halves
        // take tiles in turn)
        const int use = j - C::kStages / 2 + (values ? (two ? 2 : 1) : 0);
        if (q == 0 && j >= C::kStages / 2) ok = wait_bar(&bars.s_full[two ? use & 1 : n_sub - 1][use % kRound], (use / kRound) & 1, v);
        if (!ok) break;
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
          uint32_t y[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) y[2 * k] = e4m3x2_to_f16x2(x[p][k]), y[2 * k + 1] = e4m3x2_to_f16x2_hi(x[p][k]);
          const uint32_t at = row + (q * kPasses + p) * (kPer * 128);
          st_shared16(at + c0, make_uint4(y[0], y[1], y[2], y[3]));
          st_shared16(at + c1, make_uint4(y[4], y[5], y[6], y[7]));
        }
      }
      if (!ok) break;
      fence_proxy_async();
      mbar_arrive(&bars.full[st]);
      rs += 2, st += 2;
      if (rs >= n_raw) rs -= n_raw, rs_par ^= 1;
      if (st >= C::kStages) st -= C::kStages;
    }
  } else {
    if (kWide)
      asm volatile("setmaxnreg.dec.sync.aligned.u32 120;");
    else
      asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (w == C::kIssuer + 1 || (!kWide && w == C::kIssuer + 2)) {
      // ---------------------------------------------------------------- tiles from the cache
      // Lane g holds the page of a tile's g-th box of a page's tokens. Page ids are asked for two tiles
      // ahead and their scales one, so that no copy waits for either.
      const bool values = !kWide && w == C::kIssuer + 2;  // (codes: a warp for the keys, one for the values)
      const int log_p = v.log_page, boxes = kTok >> log_p;
      int v_exp = 127;  // exponent of the scale that those of values are relative to: the first held page's
      int page0 = 0, page1 = 0, page2 = 0;
      bool held0 = false, held1 = false, held2 = false;
      float ks0 = 0.f, vs0 = 0.f, ks1 = 0.f, vs1 = 0.f;
      auto ask_pages = [&](int j) {
        const int t = begin + j * kTok + (lane << log_p);
        // (pages wholly before the window: the table may hold anything there)
        held2 = j < n && lane < boxes && t < kv_hi && t + (1 << log_p) > walk.first;
        if (held2) page2 = kv_page_raw(v, b, t >> log_p);
      };
      auto ask_scales = [&] {
        held1 = held2, ks1 = vs1 = 0.f;
        if (held1) {
          page1 = kv_page_ok(v, page2);
          const long long at = (long long)page1 * v.heads + h;
          ks1 = v.k_scale[at], vs1 = v.v_scale[at];
        }
      };
      const char* wide = kWide ? a.wide + ((long long)(b * v.heads + h) * a.wide_tiles + begin / kTok) * (2 * C::kSlot) : nullptr;
      ask_pages(0);
      ask_scales();
      ask_pages(1);
      // the next tile's lists become the current ones, and its scales go to the softmax warps (far enough
      // ahead of them that the entry of sixteen tiles ago has been read); a scale of 0 counts as one too
      // small to matter
      auto take = [&](int j) {
        held0 = held1, page0 = page1, ks0 = ks1, vs0 = vs1;
        ask_scales();
        ask_pages(j + 2);
        if (j == 0) {
          const float ref = __shfl_sync(~0u, vs0, max(__ffs(__ballot_sync(~0u, held0)) - 1, 0));
          if (ref > 0.f) v_exp = __float_as_int(ref) >> 23 & 255;
          if (lane == 0 && !values) bars.v_ref = exp2_int(v_exp - 127);
        }
        kv_scales(v, ks0, vs0);
      };
      auto tell = [&](int j) {
        const float vs = __shfl_sync(~0u, vs0, (lane << 4) >> log_p), ks = __shfl_sync(~0u, ks0, (lane << 4) >> log_p);
        const int d = (__float_as_int(vs) >> 23) - v_exp, e = vs != 0.f ? min(max(d, -100), 100) : -100;
        if (vs != 0.f && d != e) kv_flag(v, KV_ST_SCALE);
        if (lane < 8) bars.scale[j & 15][lane] = make_float2(ks, (float)e);
        __syncwarp();
      };
      if constexpr (kWide) {
        // the first keys, then values j and keys j + 1 on one barrier: both slots are free after the same products
        constexpr int kHalf = C::kStages / 2;
        auto copy = [&](int i, uint64_t* bar) {
          bulk_g2s_at(ring_at + i % C::kStages * C::kSlot, wide + (long long)i * C::kSlot, C::kSlot, bar);
        };
        int j = -1;
        if (n > 0) {
          take(0);
          tell(0);
          if (lane == 0) mbar_expect_tx(&bars.full[0], C::kSlot), copy(0, &bars.full[0]);
          for (j = 0; j < n; ++j) {
            const bool next = j + 1 < n;
            if (next) take(j + 1);
            const int use = j - kHalf + 1;
            const bool ok = use < 0 || wait_bar(&bars.s_full[n_sub - 1][use % kRound], (use / kRound) & 1, v);
            if (!__all_sync(~0u, ok)) break;
            if (next) tell(j + 1);
            uint64_t* bar = &bars.full[1 + j % kHalf];
            if (lane == 0) {
              mbar_expect_tx(bar, (next ? 2 : 1) * C::kSlot);
              copy(2 * j + 1, bar);
              if (next) copy(2 * j + 2, bar);
            }
          }
          if (j < n)  // a wait ran out: the copies under way first (with the same limit)
            for (int k = max(0, j - kHalf); k < j; ++k) mbar_wait(&bars.full[1 + k % kHalf], (k / kHalf) & 1, kWaitLimitNs);
        }
      } else {
        int j = 0, rs = values;
        uint32_t rs_par = 1;
        for (; j < n; ++j) {
          take(j);
          const bool ok = wait_bar(&bars.raw_empty[rs], rs_par, v);
          if (!__all_sync(~0u, ok)) break;
          const uint32_t held = __ballot_sync(~0u, held0);
          if (values) {
            const float vs = __shfl_sync(~0u, vs0, (lane << 4) >> log_p);
            if (lane < 8) bars.vs[rs][lane] = vs;
            // (a group beyond kv_hi has the scale 0 too)
            const bool cut = __any_sync(~0u, lane < 8 && vs == 0.f) || begin + (j + 1) * kTok > kv_hi;
            if (lane == 0) bars.cut[rs] = cut;
            __syncwarp();
          } else {
            tell(j);
          }
          if (lane == 0) mbar_expect_tx(&bars.raw_full[rs], (uint32_t)(__popc(held) * D) << log_p);
          __syncwarp();
          if (held0)
            tma_tile(raw_slot(rs) + ((lane * D) << log_p), values ? &mv : &mk, 0, h, page0, &bars.raw_full[rs]);
          rs += 2;
          if (rs >= n_raw) rs -= n_raw, rs_par ^= 1;
        }
        if (j < n)  // a wait ran out: the copies under way first (with the same limit)
          for (int k = max(0, j - n_raw / 2); k < j; ++k)
            mbar_wait(&bars.raw_full[2 * k % n_raw + values], (2 * k / n_raw) & 1, kWaitLimitNs);
      }
    } else if (w == C::kIssuer && n > 0) {
      // ---------------------------------------------------------------- products
      // The whole warp walks, with values and conditions that are the same in every lane, so that
      // addresses and descriptors stay in uniform registers: beside eight busy softmax warps every
      // instruction between two products shows. One lane, always the same, issues.
      const int n_u = __shfl_sync(~0u, n, 0), n_sub_u = __shfl_sync(~0u, n_sub, 0);
      const bool two_u = !kWide && __shfl_sync(~0u, two, 0);
      const int step = two_u ? 2 : 1;  // from a half's tile to its next
      auto wait_all = [&](uint64_t* bar, uint32_t parity) { return __all_sync(~0u, wait_bar(bar, parity, v)) != 0; };
      constexpr uint32_t kIdS = instr_desc(kTok, false), kIdO = instr_desc(D, true);
      const uint64_t q_desc = smem_desc(q_at, 16, 1024), k_desc = smem_desc(ring_at, 16, 1024),
                     v_desc = smem_desc(ring_at, kTok * 128, 1024);
      auto qk = [&](int t, int slot) {
        const uint64_t q = q_desc + (uint32_t)((two_u ? 0 : t) * (kTileRows * D * 2 / 16)), k = k_desc + (uint32_t)(slot * (C::kSlot / 16));
        const uint32_t d = t * 128;
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
          mma_ss(d, q + ((i >> 2) * (kTileRows * 8) + (i & 3) * 2), k + ((i >> 2) * (kTok * 8) + (i & 3) * 2), kIdS, i > 0);
      };
      auto pv = [&](int t, int slot, int half, bool add) {
        const uint64_t vv = v_desc + (uint32_t)(slot * (C::kSlot / 16));
        const uint32_t d = 256 + t * 128, p = t * 128;
#pragma unroll
        for (int i = 0; i < kTok / 32; ++i)
          mma_ts(d, p + (half * (kTok / 32) + i) * 8, vv + (half * (kTok / 32) + i) * 128, kIdO, add || half || i > 0);
      };
      const bool one = elect_one();
      bool ok = wait_all(&bars.full[0], 0);
      fence_after();
      if (ok && one) {
        for (int t = 0; t < n_sub_u; ++t) {
          qk(t, 0);
          commit(&bars.s_full[t][0]);
        }
      }
      if (two_u) {
        ok = ok && wait_all(&bars.full[2], 0);
        fence_after();
        if (ok && one) {
          qk(1, 2);
          commit(&bars.s_full[1][1]);
        }
      }
      int vs = 1, ks = 2 * step % C::kStages;
      uint32_t v_par = 0, k_par = 2 * step / C::kStages;  // parities of the slots' rounds
      for (int j = 0; ok && j < n_u; ++j) {
        ok = kWide ? wait_all(&bars.full[1 + j % (C::kStages / 2)], (j / (C::kStages / 2)) & 1) : wait_all(&bars.full[vs], v_par);
        const int t_0 = two_u ? j & 1 : 0, t_n = two_u ? t_0 + 1 : n_sub_u;
        for (int t = t_0; ok && t < t_n; ++t) {
          for (int half = 0; ok && half < 2; ++half) {
            ok = wait_all(&bars.p_full[t][half], (two_u ? j >> 1 : j) & 1);
            fence_after();
            if (ok && one) pv(t, vs, half, j >= step);
          }
          if (!ok) break;
          if (one && j + step >= n_u) commit(&bars.pv_done[t]);
          if (j + step < n_u) {
            if (!kWide && t == t_0) ok = wait_all(&bars.full[ks], k_par);
            if (!ok) break;
            if (!kWide) fence_after();
            if (one) {
              qk(t, ks);
              commit(&bars.s_full[t][(j + step) % kRound]);
            }
          }
        }
        vs += 2;
        if (vs >= C::kStages) vs -= C::kStages, v_par ^= 1;
        ks += 2;
        if (ks >= C::kStages) ks -= C::kStages, k_par ^= 1;
      }
      // nothing of this block's is under way once this has arrived
      if (one) commit(&bars.end);
      wait_bar(&bars.end, 0, v);
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  fence_after();
  if (w == C::kIssuer) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// The parts of a walk, joined: a group of D / 4 lanes a row, every part's load under way at once.
template <int D, typename T>
__global__ void __launch_bounds__(256) k_kv_chunk_join(const KvAttendArgs a, int max_parts) {
  constexpr int kPart = 2 * kTileRows * (D + 4), kRowsHere = 256 / (D / 4);
  const KvView& v = a.v;
  const int h = blockIdx.x % v.heads, b = blockIdx.x / v.heads;
  pdl_trigger();
  pdl_wait();
  KvSeq s;
  if (!kv_seq(v, b, s)) return;
  const int rows = s.count * v.group;
  const int tile = (rows + 2 * kTileRows - 1) / (2 * kTileRows) - 1 - (int)blockIdx.y, r0 = tile * (2 * kTileRows);
  if (tile < 0 || rows <= a.min_rows || rows > a.max_rows) return;
  const int r_end = min(rows, r0 + 2 * kTileRows);
  const Walk walk = walk_of(a, s, r0, r_end);
  const int rr = blockIdx.z * kRowsHere + threadIdx.x / (D / 4), d = threadIdx.x % (D / 4) * 4, r = r0 + rr;
  if (walk.parts == 1 || walk.parts > max_parts || r >= r_end) return;
  const float* at = a.part + (long long)(blockIdx.y * gridDim.x + blockIdx.x) * max_parts * kPart + rr * (D + 4);
  float2 ml[kKvFan];
  float4 y[kKvFan];
#pragma unroll
  for (int i = 0; i < kKvFan; ++i)
    if (i < walk.parts) {
      ml[i] = *reinterpret_cast<const float2*>(at + (long long)i * kPart + D);
      y[i] = *reinterpret_cast<const float4*>(at + (long long)i * kPart + d);
    }
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < kKvFan; ++i)
    if (i < walk.parts) top = fmaxf(top, ml[i].x);
  const float off = top == -INFINITY ? 0.f : top;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  float lsum = 0.f;
#pragma unroll
  for (int i = 0; i < kKvFan; ++i)
    if (i < walk.parts) {
      const float f = ex2(ml[i].x - off);
      lsum = fmaf(ml[i].y, f, lsum);
      x.x = fmaf(y[i].x, f, x.x), x.y = fmaf(y[i].y, f, x.y), x.z = fmaf(y[i].z, f, x.z), x.w = fmaf(y[i].w, f, x.w);
    }
  const float inv = lsum != 0.f ? 1.f / lsum : 0.f;
  T* to = static_cast<T*>(a.out) + (long long)(s.first + r / v.group) * a.out_token + (h * v.group + r % v.group) * a.out_head + d;
  *reinterpret_cast<uint2*>(to) = make_uint2(Elem<T>::pack(x.x * inv, x.y * inv), Elem<T>::pack(x.z * inv, x.w * inv));
}

// The codes of whole sequences as halves, in the order and swizzle that the products read
// them in: [sequence][head][tile of 128 tokens][keys, values][block of 64 dimensions][token][64].
// Where many blocks walk over the same tokens, each tile is then converted once instead of by every
// one of them (a prompt of 8192 tokens 455 -> 423 us). Tokens beyond a sequence's, pages wholly before
// its window and values whose scale is 0 become 0. Bound by the latency of page, codes, store: a block for a tile's
// keys and one for its values (one for both: ragged chunks 86 us against 82).
template <int D>
__global__ void __launch_bounds__(256) k_kv_expand(const KvAttendArgs a, const uint8_t* kc, const uint8_t* vc,
                                                   long long page_stride, long long head_stride, long long token_stride) {
  constexpr int kLanes = D / 16, kPer = 256 / kLanes, kPasses = kTok / kPer, kSlot = kTok * D * 2;
  pdl_trigger();
  pdl_wait();
  const KvView& v = a.v;
  const int b = blockIdx.z, h = blockIdx.y >> 1, tile = blockIdx.x;
  const bool values = blockIdx.y & 1;
  KvSeq s;
  if (!kv_seq(v, b, s)) return;  // (the walks' kernel reports it)
  const int rows = s.count * v.group, t0 = tile * kTok;
  const int lo = a.window ? s.len - s.count - a.window + 1 : 0;  // the first token that a row sees
  if (rows <= a.min_rows || rows > a.max_rows || t0 >= s.len || t0 + kTok <= lo || tile >= a.wide_tiles) return;
  const int cl = threadIdx.x % kLanes, tk = threadIdx.x / kLanes;
  uint4 x[kPasses];
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int t = t0 + p * kPer + tk;
    x[p] = make_uint4(0, 0, 0, 0);
    if (t < s.len && (t | ((1 << v.log_page) - 1)) >= lo) {
      const int g = kv_page(v, b, t >> v.log_page);
      const long long at = g * page_stride + h * head_stride + (t & ((1 << v.log_page) - 1)) * token_stride + cl * 16;
      const float scale = values ? v.v_scale[(long long)g * v.heads + h] : 1.f;  // (beside the codes' load)
      // (not by the path for data that nothing writes while the kernel lives: it may be resident beside an
      // append that does)
      x[p] = *reinterpret_cast<const uint4*>((values ? vc : kc) + at);
      if (scale == 0.f) x[p] = make_uint4(0, 0, 0, 0);
    }
  }
  char* out = a.wide + ((long long)(b * v.heads + h) * a.wide_tiles + tile) * (2 * kSlot) + (values ? kSlot : 0);
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int tl = p * kPer + tk;
    const uint32_t ws[4] = {x[p].x, x[p].y, x[p].z, x[p].w};
    uint32_t y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[2 * i] = e4m3x2_to_f16x2(ws[i]), y[2 * i + 1] = e4m3x2_to_f16x2_hi(ws[i]);
    char* row = out + (cl >> 2) * (kTok * 128) + tl * 128;
    *reinterpret_cast<uint4*>(row + ((((cl & 3) * 2) ^ (tl & 7)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
    *reinterpret_cast<uint4*>(row + ((((cl & 3) * 2 + 1) ^ (tl & 7)) << 4)) = make_uint4(y[4], y[5], y[6], y[7]);
  }
}

template <int D, typename T, bool kWide>
cudaError_t launch(const CUtensorMap& mk, const CUtensorMap& mv, const KvAttendArgs& a, int tiles, int parts, cudaStream_t s) {
  using C = Cfg<D, kWide>;
  static std::atomic<uint64_t> seen{0};
  const cudaError_t limit = smem_limit_once(seen, reinterpret_cast<const void*>(k_kv_chunk<D, T, kWide>), C::kSmem);
  if (limit != cudaSuccess) return limit;
  return launch_pdl(k_kv_chunk<D, T, kWide>, dim3(a.v.heads * a.v.batch, tiles, parts), dim3(C::kThreads), C::kSmem, s, mk, mv, a);
}

template <int D, typename T>
cudaError_t launch_all(const CUtensorMap& mk, const CUtensorMap& mv, const KvAttendArgs& a, const fs_kv_cache& c, int tiles,
                       int parts, cudaStream_t s) {
  if (a.wide) {
    const cudaError_t e = launch_pdl(k_kv_expand<D>, dim3(a.wide_tiles, 2 * a.v.heads, a.v.batch), dim3(256), 0, s, a,
                                     static_cast<const uint8_t*>(c.k), static_cast<const uint8_t*>(c.v), (long long)c.page_stride,
                                     (long long)c.head_stride, (long long)c.token_stride);
    return e != cudaSuccess ? e : launch<D, T, true>(mk, mv, a, tiles, parts, s);
  }
  const cudaError_t e = launch<D, T, false>(mk, mv, a, tiles, parts, s);
  if (e != cudaSuccess || parts == 1) return e;
  // (blocks for the rows that a sequence can have, not for both of its tiles')
  const int rows = std::min(a.max_rows, 2 * kTileRows), here = 256 / (D / 4);
  return launch_pdl(k_kv_chunk_join<D, T>, dim3(a.v.heads * a.v.batch, tiles, (rows + here - 1) / here), dim3(256), 0, s, a, parts);
}

}  // namespace

cudaError_t launch_kv_chunk(const CUtensorMap& mk, const CUtensorMap& mv, const KvAttendArgs& a, const fs_kv_cache& c,
                            int dtype, int tiles, int parts, cudaStream_t s) {
  const bool h = dtype == FS_KV_FP16;
  if (c.dim == 128)
    return h ? launch_all<128, __half>(mk, mv, a, c, tiles, parts, s) : launch_all<128, __nv_bfloat16>(mk, mv, a, c, tiles, parts, s);
  return h ? launch_all<64, __half>(mk, mv, a, c, tiles, parts, s) : launch_all<64, __nv_bfloat16>(mk, mv, a, c, tiles, parts, s);
}

}  // namespace fs
