// Attention of a few rows over the paged 8-bit cache (single tokens, few proposals).
//
// With at most 16 rows a key head (new tokens x query heads of its group) the call
// is bound by reading the cache: 2 dim bytes a token and key head. The work is cut into
// items (sequence, key head, tile of rows) and each item's cache axis into parts, one
// block each; the blocks of a cluster join their parts through shared memory, and the last
// blocks to finish join the clusters' results (fixed order: results do not depend on which
// block is last).
//
// A warp of the block takes every fourth tile of 32 tokens and keeps kStages tiles of keys and
// values on their way into its own ring (tensor-map copies of 16 or 32 tokens of one page,
// swizzled, so that the reads below meet no bank twice); no block-wide barrier is met before the
// end. Per 16 tokens:
//   S^T [16 tokens x rows]  = K [16 x dim] Q^T          (the codes, exact in half precision)
//   O^T [dim x rows]       += V^T [dim x 16] P^T         (P rounded to half precision)
// with m16n8k16 products: tokens and dimensions fill the 16 rows of the instruction, the
// attention rows its 8 columns, so one query head costs no more padding than eight. A block takes 8
// rows, or 16 where there are more (40 rows a key head of 16 requests, which now go to k_kv_chunk, took 25 us so,
// 34 with 8 and 36 with 24, which need all registers).
// tcgen05 has nothing to add here: its smallest tile is 128 rows high, and its operands
// would have to pass through shared memory once more after the conversion.
// Three blocks an SM with two stages a warp (24 warps' rings, 192 KB an SM) read 64 sequences of up
// to 32768 tokens, 1.5 GB, in 244 us (6.3 TB/s, 92 % of the copy rate); two blocks with three
// stages took 258 us.
// The scale of a page's keys multiplies S. That of its values, a power of two relative to the
// largest met so far (v_ref), goes into P as an addend of the exponent, and m is the largest
// weight times scale: half precision's step is relative to what counts most, however far the
// scales are apart. The sum of weights is taken without it.
#include "fs_kv.cuh"

namespace fs {
namespace {

constexpr int kWarps = 4, kStages = 2, kTile = 32;
constexpr float kUp = 7.f, kSlack = 8.f;  // log2: weights are scaled by 2^kUp, and m may lag behind by kSlack: 2^15 at most

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// All blocks of the cluster that have not left (those without tokens have).
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Shared memory of the cluster's block `rank`, at this block's address a.
__device__ __forceinline__ float4 ld_cluster16(uint32_t a, int rank) {
  float4 v;
  asm volatile("{\n .reg .b32 r;\n mapa.shared::cluster.u32 r, %4, %5;\n ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [r];\n}"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(a), "r"(rank)
               : "memory");
  return v;
}
__device__ __forceinline__ float2 ld_cluster8(uint32_t a, int rank) {
  float2 v;
  asm volatile("{\n .reg .b32 r;\n mapa.shared::cluster.u32 r, %2, %3;\n ld.shared::cluster.v2.f32 {%0, %1}, [r];\n}"
               : "=f"(v.x), "=f"(v.y)
               : "r"(a), "r"(rank)
               : "memory");
  return v;
}

// Shared memory: the warps' rings of (keys, values) tiles; after the last tile the same
// bytes hold the warps' results.
template <int D>
constexpr size_t decode_smem() {
  static_assert((kWarps + 1) * 16 * D * 4 + 128 <= kWarps * kStages * 2 * kTile * D, "results fit the rings");
  return (size_t)kWarps * kStages * 2 * kTile * D + 1024;
}

template <int D, int NT, typename T>
__global__ void __launch_bounds__(kWarps * 32, D == 128 && NT == 1 ? 3 : 1)
    k_kv_decode(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, const KvAttendArgs a) {
  constexpr int kRows = 8 * NT;
  constexpr int kSteps = D / 16;   // products along the dimensions of a key
  constexpr int kMt = D / 16;      // 16-dimension tiles of O^T
  constexpr int kChunk = D / 8;    // dimensions of a value that one lane group holds
  constexpr int kTileBytes = kTile * D;
  constexpr int kPart = kRows * (D + 2);                      // floats of a partial result
  constexpr int kUnits = (kRows * (D / 4) + kWarps * 32 - 1) / (kWarps * 32);  // groups of 4 dimensions a thread joins
  extern __shared__ unsigned char raw[];
  unsigned char* ring = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
  __shared__ uint64_t bars[kWarps][kStages];
  __shared__ float sm_m[kWarps][kRows], sm_l[kWarps][kRows];
  __shared__ float2 sm_ml[kRows][kKvFan];
  __shared__ unsigned sm_last;

  const KvView& v = a.v;
  const int part = blockIdx.x, b = blockIdx.z;
  const int row_blocks = gridDim.y / v.heads;
  const int h = blockIdx.y / row_blocks, rb = blockIdx.y % row_blocks;
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tid = lane & 3;

  // before the kernel ahead in the stream has ended: nothing that it may write
  pdl_trigger();
  if (threadIdx.x < 2)  // (the copies' descriptions)
    asm volatile("prefetch.tensormap [%0];" ::"l"(threadIdx.x ? &mv : &mk) : "memory");
  if (lane == 0)
    for (int i = 0; i < kStages; ++i) mbar_init(&bars[w][i], 1);
  __syncwarp();
  pdl_wait();
  // the page of this lane's first tile, asked for before the sequence's length is known: without a
  // window the tile's place does not depend on it (entries beyond the sequence are read, not used)
  const int early_at = (part * a.split + (w + lane * kWarps) * kTile) >> v.log_page;
  int early = 0;
  if (!a.window && early_at < v.table_stride)
    asm volatile("ld.global.s32 %0, [%1];" : "=r"(early) : "l"(v.page_table + (long long)b * v.table_stride + early_at));
  KvSeq s;
  if (!kv_seq(v, b, s)) {
    if (threadIdx.x == 0 && part == 0) kv_flag(v, KV_ST_BATCH);
    return;
  }
  if (threadIdx.x == 0 && part == 0) kv_ends(v, b, s);
  const int rows = s.count * v.group;
  const int r0 = rb * kRows;
  if (r0 >= rows || rows <= a.min_rows || rows > a.max_rows) return;
  const int r_end = min(rows, r0 + kRows);
  // keys that some row of the tile sees: [kv_lo, kv_hi)
  const int pos0 = s.len - s.count + r0 / v.group, pos1 = s.len - s.count + (r_end - 1) / v.group;
  const int kv_hi = max(pos1 + 1, 0);
  const int kv_lo = a.window ? max(pos0 - a.window + 1, 0) : 0;
  const int begin = kv_lo & ~(kTile - 1);
  const int n_parts = max(1, (kv_hi - begin + a.split - 1) / a.split);
  if (n_parts > (int)gridDim.x) {  // a length beyond max_length
    if (threadIdx.x == 0 && part == 0) kv_flag(v, KV_ST_BATCH);
    return;
  }
  if (part >= n_parts) return;
  const int c0 = begin + part * a.split, c1 = min(c0 + a.split, kv_hi);
  const int n_tiles = max(0, (c1 - c0 + kTile - 1) / kTile);
  const int my_tiles = w < n_tiles ? (n_tiles - w + kWarps - 1) / kWarps : 0;

  unsigned char* my_ring = ring + w * (kStages * 2 * kTileBytes);
  // pages and scales of this warp's tiles, 32 tiles at a time, a tile a lane
  int pg0 = 0, pg1 = 0;
  float ks0 = 0.f, ks1 = 0.f, vs0 = 0.f, vs1 = 0.f;
  const bool half_tiles = v.log_page == 4;
  auto before = [&](int i) { return half_tiles && c0 + (w + i * kWarps) * kTile + 16 <= kv_lo; };
  auto load_pages = [&](int i0) {
    const int i = i0 + lane;
    pg0 = pg1 = 0;
    ks0 = ks1 = vs0 = vs1 = 0.f;
    if (i < my_tiles) {
      const int t = c0 + (w + i * kWarps) * kTile;
      // (a tile's first page may lie wholly before the window, where the table may hold anything: the second
      // is taken twice, and the values' scale below says 0)
      pg0 = pg1 = !a.window && i0 == 0 ? kv_page_ok(v, early) : kv_page(v, b, (t + (before(i) ? 16 : 0)) >> v.log_page);
      if (half_tiles && t + 16 < s.len) pg1 = kv_page(v, b, (t + 16) >> v.log_page);
    }
  };
  auto load_scales = [&](int i0) {
    if (i0 + lane < my_tiles) {
      const long long at0 = (long long)pg0 * v.heads + h, at1 = (long long)pg1 * v.heads + h;
      ks0 = v.k_scale[at0], vs0 = v.v_scale[at0];
      ks1 = ks0, vs1 = vs0;
      if (pg1 != pg0) ks1 = v.k_scale[at1], vs1 = v.v_scale[at1];
      if (before(i0 + lane)) vs0 = 0.f;
    }
  };
  // one of a tile's copies into its stage: keys, values, and those of the second page
  auto copy = [&](int i, int which, int p0, int p1) {
    const int st = i % kStages, t = c0 + (w + i * kWarps) * kTile, slot = t & ((1 << v.log_page) - 1);
    tma_tile(smem_u32(my_ring) + st * (2 * kTileBytes) + (which & 1) * kTileBytes + (which >> 1) * (kTileBytes / 2),
             which & 1 ? &mv : &mk, half_tiles ? 0 : slot, h, which >> 1 ? p1 : p0, &bars[w][st]);
  };
  auto issue = [&](int i, int p0, int p1) {
    if (lane == 0) mbar_expect_tx(&bars[w][i % kStages], 2 * kTileBytes);
    __syncwarp();
    if (lane < (half_tiles ? 4 : 2)) copy(i, lane, p0, p1);
  };

  // queries' loads first, then the first copies: the lanes of a stage issue its own
  uint4 qraw[NT][kSteps / 4][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = r0 + n * 8 + gid;
    const T* q = static_cast<const T*>(a.q) + (long long)(s.first + r / v.group) * a.q_token +
                 (h * v.group + r % v.group) * a.q_head;
#pragma unroll
    for (int c = 0; c < kSteps / 4; ++c)
#pragma unroll
      for (int k = 0; k < 2; ++k)
        qraw[n][c][k] = r < r_end ? *reinterpret_cast<const uint4*>(q + (tid * (kSteps / 4) + c) * 16 + 8 * k) : make_uint4(0, 0, 0, 0);
  }
  load_pages(0);
  {
    const int i = lane >> 2, p0 = __shfl_sync(~0u, pg0, i), p1 = __shfl_sync(~0u, pg1, i);
    const bool mine = i < kStages && i < my_tiles;
    if (mine && (lane & 3) == 0) mbar_expect_tx(&bars[w][i], 2 * kTileBytes);
    __syncwarp();
    if (mine && (lane & 3) < (half_tiles ? 4 : 2)) copy(i, lane & 3, p0, p1);
  }
  load_scales(0);

  // queries: row gid of each tile of 8 rows, in the order that the codes come in
  uint32_t qf[NT][kSteps][2];
  float cq[NT][2];  // of rows 2 tid, 2 tid + 1: the row's power of two, the scale, log2(e)
  int hi_lim[NT][2], lo_lim[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float f[kSteps * 4];
    float amax = 0.f;
#pragma unroll
    for (int c = 0; c < kSteps / 4; ++c) {
      const uint4 x = qraw[n][c][0], y = qraw[n][c][1];
      const uint32_t u[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 z = Elem<T>::two(u[i]);
        f[c * 16 + 2 * i] = z.x, f[c * 16 + 2 * i + 1] = z.y;
        amax = fmaxf(amax, fmaxf(fabsf(z.x), fabsf(z.y)));
      }
    }
    amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 2));
    const int e = row_exponent(amax);
    const float down = exp2_int(-e);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      qf[n][i][0] = pack_f16(f[4 * i] * down, f[4 * i + 1] * down);
      qf[n][i][1] = pack_f16(f[4 * i + 2] * down, f[4 * i + 3] * down);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      cq[n][j] = a.scale_log2 * exp2_int(__shfl_sync(~0u, e, (2 * tid + j) * 4));
      const int rj = r0 + n * 8 + 2 * tid + j;
      const int pos = s.len - s.count + rj / v.group;
      hi_lim[n][j] = rj < r_end ? pos : -1;
      lo_lim[n][j] = a.window ? pos - a.window + 1 : 0;
    }
  }
  // tiles inside [full_lo, full_hi) are seen whole by every row
  const int full_hi = pos0 + 1;
  const int full_lo = a.window ? pos1 - a.window + 1 : 0;

  float o[kMt][NT][4];
  float m[NT][2], l[NT][2], v_ref = 0.f;
#pragma unroll
  for (int j = 0; j < kMt; ++j)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[j][n][i] = 0.f;
#pragma unroll
  for (int n = 0; n < NT; ++n) m[n][0] = m[n][1] = -INFINITY, l[n][0] = l[n][1] = 0.f;

  bool ok = true;
  int done = 0;
  for (int i = 0; i < my_tiles; done = ++i) {
    if ((i & 31) == 0) {
      if (i) {
        // (tiles already under way took their pages from the lists of the round before)
        load_pages(i);
        load_scales(i);
      }
      kv_scales(v, ks0, vs0);
      kv_scales(v, ks1, vs1);
      float top = fmaxf(vs0, vs1);
#pragma unroll
      for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
      if (top > v_ref) {
        // weights times scales, and their maxima, are relative to v_ref; the sums of weights are not
        if (v_ref > 0.f) {
          const int up = min((__float_as_int(top) >> 23) - (__float_as_int(v_ref) >> 23), 100);
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int k = 0; k < 2; ++k) m[n][k] -= (float)up, l[n][k] = fminf(l[n][k] * exp2_int(up), 0x1p120f);
        }
        v_ref = top;
      }
    }
    const int st = i % kStages, t0 = c0 + (w + i * kWarps) * kTile;
    const float ks[2] = {__shfl_sync(~0u, ks0, i & 31), __shfl_sync(~0u, ks1, i & 31)};
    // log2 of the values' scale over the largest so far; a scale of 0 counts as one too small to
    // matter, and its values as 0
    const float vs[2] = {__shfl_sync(~0u, vs0, i & 31), __shfl_sync(~0u, vs1, i & 31)};
    int ve[2];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
      ve[mt] = vs[mt] != 0.f ? max((__float_as_int(vs[mt]) >> 23) - (__float_as_int(v_ref) >> 23), -100) : -100;
    ok = mbar_wait(&bars[w][st], (i / kStages) & 1, kWaitLimitNs);
    if (!__all_sync(~0u, ok)) break;
    const unsigned char* kt = my_ring + st * (2 * kTileBytes);
    const unsigned char* vt = kt + kTileBytes;

    float sc[2][NT][4];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      float sc1[NT][4];  // (two chains of products: half the latency)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < 4; ++k) sc[mt][n][k] = sc1[n][k] = 0.f;
#pragma unroll
      for (int c = 0; c < kSteps / 4; ++c) {
        // 16 codes of tokens gid and gid + 8
        const int chunk = D == 128 ? (2 * tid + c) ^ gid : tid ^ (gid >> 1);
        const unsigned char* at = kt + (mt * 16 + gid) * D + chunk * 16;
        const uint4 x = *reinterpret_cast<const uint4*>(at), y = *reinterpret_cast<const uint4*>(at + 8 * D);
        const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t a0 = e4m3x2_to_f16x2(xs[k]), a2 = e4m3x2_to_f16x2_hi(xs[k]);
          const uint32_t a1 = e4m3x2_to_f16x2(ys[k]), a3 = e4m3x2_to_f16x2_hi(ys[k]);
#pragma unroll
          for (int n = 0; n < NT; ++n) mma16816(k & 1 ? sc1[n] : sc[mt][n], a0, a1, a2, a3, qf[n][c * 4 + k][0], qf[n][c * 4 + k][1]);
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < 4; ++k) sc[mt][n][k] += sc1[n][k];
    }
    const bool whole = t0 >= full_lo && t0 + kTile <= full_hi;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float x = fmaf(sc[mt][n][k], ks[mt] * cq[n][k & 1], (float)ve[mt]);
          if (!whole) {
            const int t = t0 + mt * 16 + gid + (k >> 1) * 8;
            if (t > hi_lim[n][k & 1] || t < lo_lim[n][k & 1]) x = -INFINITY;
          }
          sc[mt][n][k] = x;
        }
    // m, the reference of the weights, follows the rows' maxima only when one of them has grown by
    // more than 2^kSlack: most tiles need no exchange between lanes. A row without a key yet keeps
    // -infinity, and 0 in its place.
    float lm[NT][2];
    bool grow = false;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        lm[n][j] = fmaxf(fmaxf(sc[0][n][j], sc[0][n][j + 2]), fmaxf(sc[1][n][j], sc[1][n][j + 2]));
        grow |= lm[n][j] > m[n][j] + kSlack || (m[n][j] == -INFINITY && lm[n][j] > m[n][j]);
      }
    if (__any_sync(~0u, grow)) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float corr[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float x = lm[n][j];
          x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
          x = fmaxf(x, __shfl_xor_sync(~0u, x, 8));
          x = fmaxf(x, __shfl_xor_sync(~0u, x, 16));
          const float m_new = fmaxf(m[n][j], x);
          corr[j] = ex2(m[n][j] - (m_new == -INFINITY ? 0.f : m_new));
          m[n][j] = m_new;
          l[n][j] *= corr[j];
        }
#pragma unroll
        for (int j = 0; j < kMt; ++j) {
          o[j][n][0] *= corr[0], o[j][n][2] *= corr[0];
          o[j][n][1] *= corr[1], o[j][n][3] *= corr[1];
        }
      }
    }
    uint32_t pf[2][NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float up[2] = {(m[n][0] == -INFINITY ? 0.f : m[n][0]) - kUp, (m[n][1] == -INFINITY ? 0.f : m[n][1]) - kUp};
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float p0 = ex2(sc[mt][n][2 * k] - up[0]), p1 = ex2(sc[mt][n][2 * k + 1] - up[1]);
          l[n][0] = fmaf(p0, exp2_int(-ve[mt]), l[n][0]), l[n][1] = fmaf(p1, exp2_int(-ve[mt]), l[n][1]);
          pf[mt][n][k] = transpose8x8(pack_f16(p0, p1));
        }
    }
    const bool tail = t0 + kTile > s.len;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      // codes of tokens 2 tid, 2 tid + 1, 2 tid + 8, 2 tid + 9: kChunk dimensions from gid * kChunk on
      uint32_t vw[4][kChunk / 4];
#pragma unroll
      for (int i2 = 0; i2 < 4; ++i2) {
        const int t = mt * 16 + 2 * tid + (i2 & 1) + (i2 >> 1) * 8;
        if constexpr (D == 128) {
          const uint4 x = *reinterpret_cast<const uint4*>(vt + t * D + ((gid ^ (t & 7)) * 16));
          vw[i2][0] = x.x, vw[i2][1] = x.y, vw[i2][2] = x.z, vw[i2][3] = x.w;
        } else {
          const uint2 x = *reinterpret_cast<const uint2*>(vt + t * D + (((gid >> 1) ^ ((t >> 1) & 3)) * 16) + (gid & 1) * 8);
          vw[i2][0] = x.x, vw[i2][1] = x.y;
        }
        if ((tail && t0 + t >= s.len) || vs[mt] == 0.f) {  // slots without a token may hold NaN codes
#pragma unroll
          for (int k = 0; k < kChunk / 4; ++k) vw[i2][k] = 0;
        }
      }
#pragma unroll
      for (int k = 0; k < kChunk / 4; ++k) {
        const uint32_t u0 = __byte_perm(vw[0][k], vw[1][k], 0x5140), u1 = __byte_perm(vw[0][k], vw[1][k], 0x7362);
        const uint32_t x0 = __byte_perm(vw[2][k], vw[3][k], 0x5140), x1 = __byte_perm(vw[2][k], vw[3][k], 0x7362);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma16816(o[2 * k][n], e4m3x2_to_f16x2(u0), e4m3x2_to_f16x2_hi(u0), e4m3x2_to_f16x2(x0), e4m3x2_to_f16x2_hi(x0),
                   pf[mt][n][0], pf[mt][n][1]);
          mma16816(o[2 * k + 1][n], e4m3x2_to_f16x2(u1), e4m3x2_to_f16x2_hi(u1), e4m3x2_to_f16x2(x1),
                   e4m3x2_to_f16x2_hi(x1), pf[mt][n][0], pf[mt][n][1]);
        }
      }
    }
    __syncwarp();  // every lane has read the stage
    // the next tile of this stage; its pages are in the lists of its round of 32
    const int nx = i + kStages;
    if (nx < my_tiles) {
      int p0, p1;
      if ((nx & ~31) == (i & ~31)) {
        p0 = __shfl_sync(~0u, pg0, nx & 31), p1 = __shfl_sync(~0u, pg1, nx & 31);
      } else {
        const int t = c0 + (w + nx * kWarps) * kTile;
        p0 = p1 = kv_page(v, b, t >> v.log_page);
        if (half_tiles && t + 16 < s.len) p1 = kv_page(v, b, (t + 16) >> v.log_page);
      }
      issue(nx, p0, p1);
    }
  }
  if (!__all_sync(~0u, ok)) {
    // give up: say so, and wait (with the same limit) for the copies still under way
    if (lane == 0) kv_flag(v, ST_TIMEOUT);
    for (int i = done; i < min(done + kStages, my_tiles); ++i)
      mbar_wait(&bars[w][i % kStages], (i / kStages) & 1, kWaitLimitNs);
  }

  // ---- join the warps
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) l[n][j] += __shfl_xor_sync(~0u, l[n][j], d);
      if (gid == 0) sm_m[w][n * 8 + 2 * tid + j] = m[n][j], sm_l[w][n * 8 + 2 * tid + j] = l[n][j];
    }
  __syncthreads();  // every warp has left its ring
  float* ow = reinterpret_cast<float*>(ring);  // [kWarps][kRows][D]
#pragma unroll
  for (int j = 0; j < kMt; ++j)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        // rows gid, gid + 8 of tile j are dimensions gid * kChunk + 2 j, + 1
        const int r = n * 8 + 2 * tid + k;
        *reinterpret_cast<float2*>(ow + ((w * kRows + r) * D + gid * kChunk + 2 * j)) =
            make_float2(o[j][n][k] * v_ref, o[j][n][k + 2] * v_ref);
      }
  __syncthreads();

  const int n_rows = r_end - r0;
  const long long item = ((long long)b * gridDim.y + blockIdx.y);
  // the blocks of a cluster hold consecutive parts of one item; `active` of them have tokens
  const int rank = part % a.cluster, active = min(a.cluster, n_parts - (part - rank));
  float* part_o = a.part + (item * gridDim.x + (part - rank)) * kPart;  // the cluster's result
  float* res = ow + kWarps * kRows * D;                                 // this block's, for its cluster
  auto write_out = [&](int r, int d, float4 x, float lsum) {
    const float inv = lsum > 0.f ? 1.f / lsum : 0.f;
    const int rr = r0 + r;
    T* to = static_cast<T*>(a.out) + (long long)(s.first + rr / v.group) * a.out_token +
            (h * v.group + rr % v.group) * a.out_head + d;
    *reinterpret_cast<uint2*>(to) = make_uint2(Elem<T>::pack(x.x * inv, x.y * inv), Elem<T>::pack(x.z * inv, x.w * inv));
  };
  for (int u = threadIdx.x; u < n_rows * (D / 4); u += kWarps * 32) {
    const int r = u / (D / 4), d = u % (D / 4) * 4;
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) top = fmaxf(top, sm_m[i][r]);
    const float base = top == -INFINITY ? 0.f : top;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    float lsum = 0.f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      const float f = ex2(sm_m[i][r] - base);
      const float4 y = *reinterpret_cast<const float4*>(ow + (i * kRows + r) * D + d);
      lsum = fmaf(sm_l[i][r], f, lsum);
      x.x = fmaf(y.x, f, x.x), x.y = fmaf(y.y, f, x.y), x.z = fmaf(y.z, f, x.z), x.w = fmaf(y.w, f, x.w);
    }
    if (n_parts == 1) {
      write_out(r, d, x, lsum);
    } else if (active > 1) {
      *reinterpret_cast<float4*>(res + r * D + d) = x;
      if (d == 0) *reinterpret_cast<float2*>(res + kRows * D + 2 * r) = make_float2(top, lsum);
    } else {
      *reinterpret_cast<float4*>(part_o + r * D + d) = x;
      if (d == 0) *reinterpret_cast<float2*>(part_o + kRows * D + 2 * r) = make_float2(top, lsum);
    }
  }
  if (n_parts == 1) return;

  // ---- join the cluster's parts, each of its blocks a share of the rows' dimensions
  if (active > 1) {
    cluster_sync();
    const uint32_t res_at = smem_u32(res);
    for (int u = rank * kWarps * 32 + threadIdx.x; u < n_rows * (D / 4); u += active * kWarps * 32) {
      const int r = u / (D / 4), d = u % (D / 4) * 4;
      float2 ml[kKvCluster];
      float4 y[kKvCluster];
#pragma unroll
      for (int i = 0; i < kKvCluster; ++i)
        if (i < active) {
          ml[i] = ld_cluster8(res_at + 4 * (kRows * D + 2 * r), i);
          y[i] = ld_cluster16(res_at + 4 * (r * D + d), i);
        }
      float top = -INFINITY, lsum = 0.f;
#pragma unroll
      for (int i = 0; i < kKvCluster; ++i)
        if (i < active) top = fmaxf(top, ml[i].x);
      const float base = top == -INFINITY ? 0.f : top;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kKvCluster; ++i)
        if (i < active) {
          const float f = ex2(ml[i].x - base);
          lsum = fmaf(ml[i].y, f, lsum);
          x.x = fmaf(y[i].x, f, x.x), x.y = fmaf(y[i].y, f, x.y), x.z = fmaf(y[i].z, f, x.z), x.w = fmaf(y[i].w, f, x.w);
        }
      if (active == n_parts) {
        write_out(r, d, x, lsum);
      } else {
        *reinterpret_cast<float4*>(part_o + r * D + d) = x;
        if (d == 0) *reinterpret_cast<float2*>(part_o + kRows * D + 2 * r) = make_float2(top, lsum);
      }
    }
    cluster_sync();  // no block leaves while another reads its shared memory
    if (active == n_parts || rank) return;
  }

  // ---- join the clusters' results: the last block of every kKvFan, then the last of those
  float* parts = a.part + item * gridDim.x * kPart;
  // of `count` results, `step` parts apart, mine is the `me`-th
  int me = part / a.cluster, count = (n_parts + a.cluster - 1) / a.cluster, step = a.cluster;
  unsigned* ticket = a.ticket + item * a.tickets;
  for (bool first = a.tickets > 1;; first = false) {
    const int g = first ? me / kKvFan : 0, g0 = first ? g * kKvFan : 0, g_n = first ? min(kKvFan, count - g0) : count;
    __syncthreads();
    if (threadIdx.x == 0) {
      __threadfence();  // (the block's results, ordered before by the barrier, become visible with the ticket)
      unsigned* at = ticket + (first ? 1 + g : 0);
      const unsigned t = atomicAdd(at, 1u);
      sm_last = t == (unsigned)g_n - 1;
      if (sm_last) *at = 0;  // as it was found
      __threadfence();
    }
    __syncthreads();
    if (!sm_last) return;
    const bool done = g_n == count;  // nothing is left to join with
    float* from = parts + (long long)(g0 * step) * kPart;
    // sixteen results at a time, every load of a unit under way at once, the first unit's beside
    // those of the weights
    float4 acc[kUnits];
    float lsum[kUnits], top[kUnits];
#pragma unroll
    for (int i = 0; i < kUnits; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f), lsum[i] = 0.f, top[i] = -INFINITY;
    for (int i0 = 0; i0 < g_n; i0 += kKvFan) {
      const int m_n = min(kKvFan, g_n - i0);
      float4 y[kKvFan];
      auto load = [&](int k) {
        const int u = threadIdx.x + k * kWarps * 32, r = u / (D / 4), d = u % (D / 4) * 4;
#pragma unroll
        for (int i = 0; i < kKvFan; ++i)
          if (i < m_n && r < n_rows)
            y[i] = __ldcg(reinterpret_cast<const float4*>(from + (long long)((i0 + i) * step) * kPart + r * D + d));
      };
      load(0);
      if (i0) __syncthreads();
      for (int u = threadIdx.x; u < kRows * kKvFan; u += kWarps * 32) {
        const int r = u / kKvFan, i = u % kKvFan;
        float2 ml = make_float2(-INFINITY, 0.f);
        if (i < m_n && r < n_rows)
          ml = __ldcg(reinterpret_cast<const float2*>(from + (long long)((i0 + i) * step) * kPart + kRows * D + 2 * r));
        sm_ml[r][i] = ml;
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kUnits; ++k) {
        const int u = threadIdx.x + k * kWarps * 32, r = u / (D / 4);
        if (k) load(k);
        if (r >= n_rows) continue;
        float m_new = top[k];
#pragma unroll
        for (int i = 0; i < kKvFan; ++i) m_new = fmaxf(m_new, sm_ml[r][i].x);
        const float base = m_new == -INFINITY ? 0.f : m_new, f0 = ex2(top[k] - base);
        top[k] = m_new, lsum[k] *= f0;
        acc[k].x *= f0, acc[k].y *= f0, acc[k].z *= f0, acc[k].w *= f0;
#pragma unroll
        for (int i = 0; i < kKvFan; ++i)
          if (i < m_n) {
            const float f = ex2(sm_ml[r][i].x - base);
            lsum[k] = fmaf(sm_ml[r][i].y, f, lsum[k]);
            acc[k].x = fmaf(y[i].x, f, acc[k].x), acc[k].y = fmaf(y[i].y, f, acc[k].y);
            acc[k].z = fmaf(y[i].z, f, acc[k].z), acc[k].w = fmaf(y[i].w, f, acc[k].w);
          }
      }
    }
    if (!done) __syncthreads();  // (every maximum and sum has been read)
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
      const int u = threadIdx.x + k * kWarps * 32, r = u / (D / 4), d = u % (D / 4) * 4;
      if (r >= n_rows) continue;
      if (done) {
        write_out(r, d, acc[k], lsum[k]);
      } else {  // in the place of the first of them
        *reinterpret_cast<float4*>(from + r * D + d) = acc[k];
        if (d == 0) *reinterpret_cast<float2*>(from + kRows * D + 2 * r) = make_float2(top[k], lsum[k]);
      }
    }
    if (done) return;
    me = g, count = (count + kKvFan - 1) / kKvFan, step *= kKvFan;
  }
}

template <int D, int NT, typename T>
cudaError_t launch(const CUtensorMap& mk, const CUtensorMap& mv, const KvAttendArgs& a, int row_blocks, int splits,
                   cudaStream_t s) {
  static std::atomic<uint64_t> seen{0};
  const cudaError_t limit = smem_limit_once(seen, reinterpret_cast<const void*>(k_kv_decode<D, NT, T>), decode_smem<D>());
  if (limit != cudaSuccess) return limit;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((splits + a.cluster - 1) / a.cluster * a.cluster, a.v.heads * row_blocks, a.v.batch);
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = decode_smem<D>();
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {(unsigned)a.cluster, 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = a.cluster > 1 ? 2 : 1;
  note_launch();
  return cudaLaunchKernelEx(&cfg, k_kv_decode<D, NT, T>, mk, mv, a);
}

template <int D, typename T>
cudaError_t launch_rows(const CUtensorMap& mk, const CUtensorMap& mv, const KvAttendArgs& a, int row_tile,
                        int row_blocks, int splits, cudaStream_t s) {
  return row_tile == 8 ? launch<D, 1, T>(mk, mv, a, row_blocks, splits, s) : launch<D, 2, T>(mk, mv, a, row_blocks, splits, s);
}

}  // namespace

cudaError_t launch_kv_decode(const CUtensorMap& mk, const CUtensorMap& mv, const KvAttendArgs& a, int dim, int dtype,
                             int row_tile, int row_blocks, int splits, cudaStream_t s) {
  const bool h = dtype == FS_KV_FP16;
  if (dim == 128)
    return h ? launch_rows<128, __half>(mk, mv, a, row_tile, row_blocks, splits, s)
             : launch_rows<128, __nv_bfloat16>(mk, mv, a, row_tile, row_blocks, splits, s);
  return h ? launch_rows<64, __half>(mk, mv, a, row_tile, row_blocks, splits, s)
           : launch_rows<64, __nv_bfloat16>(mk, mv, a, row_tile, row_blocks, splits, s);
}

}  // namespace fs
