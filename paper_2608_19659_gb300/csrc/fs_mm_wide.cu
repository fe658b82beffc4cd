// Products of many rows: pairs of SMs on tiles of 256 rows and 64 to 256 columns, tcgen05.
//
// A cluster of two blocks holds a tile: each block loads its 128 rows of A and its 128 of B (half of what one SM
// alone would read for a tile of that shape), one thread of the first issues the products of both
// (cta_group::2), and each block has its 128 rows' 256 sums in its tensor memory, twice: while eight warps finish a tile and store
// it, the next one's sums are under way. Blocks stay for the whole launch and walk over the tiles, eight tiles of rows wide,
// so that what is resident at a time shares its rows of W through the L2.
// A launch holds up to three products (the backward pass: dx and both dW), whose sums may have up to four parts (dx: over gate
// and up, each of one term or two) and whose operands may lie either way (dx reads W, dW reads both, across their rows).
// Of a gated block the first SM of a pair loads gate's rows and the second up's, so that a thread has both sums of a result.
// Bound by the tensor cores, and they by power: 8192 rows of 8192 bf16 over 10240 677 to 690 us in a burst (2.0 PFLOP/s), 750 to 790 in a
// row; 4096 rows of 7168 8-bit over 8192 131 us (3.7); the tensor pipe is active 87 to 90 % of the time with full waves. Tiles of short
// sums are bound by their end (4096 rows of 1024 8-bit terms over 8192 columns 33 us, with a residual 48; the products alone 16): a tile's
// takes 2.5 us, of a residual and an activation up to 5.5.
#include <algorithm>
#include <atomic>
#include <cfloat>
#include <utility>

#include "fs_mm.cuh"

namespace fs {
namespace {

constexpr int kStages = 8, kHalf = 128 * kMmBlock, kRing = 12 * kHalf;  // (stages at most)
constexpr int kTile = kWideTile;            // rows of a tile; its columns at most
constexpr int kGroup = 8;  // tiles of rows that are walked over together (4, 12 and 16 are 1 to 4 % slower)

constexpr int kThreads = 12 * 32, kEnders = 8;  // (warps that finish tiles: two for each of the four groups of 32 rows)

struct WideBars {
  uint64_t full[kStages], empty[kStages], sum_full[2], sum_empty[2];
  uint32_t tmem;
  alignas(16) float scale[kTile];  // of a tile's columns of W (gated: gate's, then up's)
  uint16_t bias[kTile];
  alignas(16) uint4 pass[kEnders][32 * 4];  // of each warp that finishes tiles: 32 rows' 64 bytes, on their way from or to memory
};
// All of an SM's shared memory: no block with tensor memory of its own fits beside one of these, which
// take all of it. (One that held some while it waits for its cluster, and this pair for each other: none would go on.)
constexpr size_t kSmem = 226 * 1024;
static_assert(kSmem >= 1024 + kRing + sizeof(WideBars), "a block's shared memory");

constexpr int kParts = 4;  // of a gradient's sum, at most

// Whether a tile's columns are W's rows (and not gate's and up's).
__host__ __device__ constexpr bool one_sum(int mode) { return mode == MM_LINEAR || mode == MM_GRAD; }

// One tile: of product q, rows from m0 and columns (gated: results) from n0.
struct Tile {
  int q, m0, n0;
};
// (never by a pointer: what a kernel's arguments hold is read by its index, or for a single product as constants)
template <int kMode>
__device__ __forceinline__ const MmProduct& product_of(const MmWideArgs& a, const Tile& t) {
  return a.product[kMode == MM_GRAD ? t.q : 0];
}

template <int kMode>
__device__ __forceinline__ Tile tile_of(const MmWideArgs& a, int i) {
  Tile t{};
  if (kMode == MM_GRAD)
    while (t.q + 1 < a.products && i >= a.product[t.q].tiles) i -= a.product[t.q++].tiles;
  const MmProduct& p = product_of<kMode>(a, t);
  const int g = (int)((unsigned)i / (unsigned)p.group), r = i - g * p.group, high = min(kGroup, p.row_tiles - g * kGroup);
  const int across = high == kGroup ? r / kGroup : (int)((unsigned)r / (unsigned)high);
  t.m0 = (g * kGroup + r - across * high) * kTile;
  t.n0 = across * (one_sum(kMode) ? p.tile : p.tile / 2);
  return t;
}

__device__ __forceinline__ void tma_pair(uint32_t dst, const CUtensorMap* m, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(m), "r"(x), "r"(y), "r"(bar)
      : "memory");
}
template <bool kEight>
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  if constexpr (kEight)
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
// Arrives on both blocks' barrier once the products issued so far are done.
__device__ __forceinline__ void commit_pair(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
               "h"((uint16_t)3)
               : "memory");
}
__device__ __forceinline__ void arrive_at(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// Eight neighbouring 16-bit values of a row, n of them inside it (others 0).
__device__ __forceinline__ uint4 load8(const void* row, long long at, int n) {
  const uint16_t* p = static_cast<const uint16_t*>(row) + at;
  if (n >= 8) return *reinterpret_cast<const uint4*>(p);
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) w[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(void* row, long long at, uint4 v, int n) {
  uint16_t* p = static_cast<uint16_t*>(row) + at;
  if (n >= 8) {
    *reinterpret_cast<uint4*>(p) = v;
    return;
  }
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
}
template <typename T>
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  return make_uint4(Elem<T>::pack(v[0], v[1]), Elem<T>::pack(v[2], v[3]), Elem<T>::pack(v[4], v[5]), Elem<T>::pack(v[6], v[7]));
}
__device__ __forceinline__ void tmem_ld(uint32_t (&r)[32], uint32_t a) { tmem_ld32(r, a); }
__device__ __forceinline__ void tmem_ld(uint32_t (&r)[16], uint32_t a) { tmem_ld16(r, a); }
template <typename T>
__device__ __forceinline__ void floats8(float (&v)[8], uint4 w) {
  const float2 a = Elem<T>::two(w.x), b = Elem<T>::two(w.y), c = Elem<T>::two(w.z), d = Elem<T>::two(w.w);
  v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y, v[4] = c.x, v[5] = c.y, v[6] = d.x, v[7] = d.y;
}
// What rounding v to w left, rounded in its turn.
template <typename T>
__device__ __forceinline__ uint4 left8(const float (&v)[8], uint4 w) {
  float r[8];
  floats8<T>(r, w);
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = v[j] - r[j];
  return pack8<T>(r);
}
__device__ __forceinline__ void floats8(float (&v)[8], const float* p) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}

template <typename T, int kMode>
__global__ void __launch_bounds__(kThreads, 1) k_mm_wide(const __grid_constant__ MmWideArgs a) {
  extern __shared__ unsigned char raw[];
  const uint32_t smem = (smem_u32(raw) + 1023) & ~1023u;
  WideBars& bars = *reinterpret_cast<WideBars*>(raw + (smem - smem_u32(raw)) + kRing);
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  // This pair's tiles: every `step`-th. Of gradients whose longest tiles are fewer than there are pairs, those pairs start with one of them, as
  // long as `rounds` of the others, which the other pairs take meanwhile: then `next` is the k-th tile.
  const int first = blockIdx.x >> 1, step = gridDim.x >> 1;
  auto next = [&](int i, int k) { return kMode == MM_GRAD ? mm_next_tile(i, k, first, step, a.lead, a.rounds) : i + step; };

  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int i = 0; i < a.stages; ++i) mbar_init(&bars.full[i], 1), mbar_init(&bars.empty[i], 1);
    for (int i = 0; i < 2; ++i) mbar_init(&bars.sum_full[i], 1), mbar_init(&bars.sum_empty[i], 2 * kEnders);
  }
  if (w == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&bars.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  pdl_wait();
  __syncwarp();
  fence_before();
  cluster_all();
  fence_after();
  constexpr uint32_t tmem = 0;  // (all of tensor memory is this block's: its columns begin at 0)

  // Copies and products: the whole warp walks, with values that are the same in every lane, so that addresses and descriptors stay
  // in uniform registers; one lane, always the same, issues.
  if (w == 0 || w == 2) {
    // ---------------------------------------------------------------- copies: a warp for A, one for B
    const bool of_b = w == 2, one = elect_one();
    if (one) fence_proxy_async_all();
    const int per = a.eight ? kMmBlock : kMmBlock / 2;
    const uint32_t leader = cluster_addr(smem_u32(&bars.full[0]), 0), ring = smem + (of_b ? a.sub * kHalf : 0);
    const int stages = a.stages, stage = a.stage;
    int st = 0, count = 0;
    uint32_t par = 1, at = ring;
    bool ok = true;
    const bool two = a.sub == 2;
    // the blocks of one part of a tile's sum, of rows from `row` on
    auto copy = [&](auto mn, const CUtensorMap* map, int row, int end, uint32_t part_bytes, uint32_t bytes, bool high) {
      auto block = [&](uint32_t to, int x, uint32_t bar) {
        if constexpr (decltype(mn)::value) {
          tma_pair(to, map, row, x, bar);
          if (high) tma_pair(to + kHalf / 2, map, row + 64, x, bar);
        } else {
          tma_pair(to, map, x, row, bar);
        }
      };
      for (int x = 0; x < end; x += two ? 2 * per : per) {
        ok = mm_wait(&bars.empty[st], par, a.status);
        if (!ok) break;
        if (one) {
          const uint32_t bar = leader + st * 8;
          // (B's bytes may be counted before they are expected: the arrival that goes with that is still to come)
          if (!of_b && rank == 0) mbar_expect_tx(&bars.full[st], bytes);
          block(at, x, bar);
          if (two) block(at + part_bytes, x + per, bar);  // (beyond the sum's end: filled with zeros)
        }
        count = min(count + 1, stages);
        at += stage;
        if (++st == stages) st = 0, par ^= 1, at = ring;
      }
    };
    int n = 0;
    for (int i = first; ok && i < a.tiles; i = next(i, ++n)) {
      const Tile t = tile_of<kMode>(a, i);
      const MmProduct& p = product_of<kMode>(a, t);
      const int row = !of_b ? t.m0 + rank * 128 : one_sum(kMode) ? t.n0 + rank * (p.tile / 2) : t.n0;
      const uint32_t part_bytes = of_b ? p.tile / 2 * kMmBlock : kHalf, bytes = a.sub * (2 * kHalf + p.tile * kMmBlock);  // a block's; both SMs' stage
      const bool high = !of_b || p.tile > 128;
      for (int part = 0; ok && part < (kMode == MM_GRAD ? kParts : 1); ++part) {
        const CUtensorMap* map = &a.maps[of_b ? p.b[one_sum(kMode) ? part : rank] : p.a[part]];
        const int end = p.blocks[part] * per;
        if (kMode == MM_GRAD && (of_b ? p.b_mn : p.a_mn))
          copy(std::true_type(), map, row, end, part_bytes, bytes, high);
        else
          copy(std::false_type(), map, row, end, part_bytes, bytes, high);
      }
    }
    if (ok) {
      // every slot's last products are done, and their arrivals here have come
      for (int j = 0; j < count; ++j) {
        if (--st < 0) st = a.stages - 1, par ^= 1;
        mm_wait(&bars.empty[st], par ^ 1, a.status);
      }
    } else {
      // a wait ran out: the copies under way end within microseconds
      const uint64_t t0 = global_ns();
      for (int j = 0; j < (1 << 20) && global_ns() - t0 < 1000000; ++j) {
      }
    }
  } else if (w == 1 && rank == 0) {
    // ---------------------------------------------------------------- products of both blocks
    const bool one = elect_one();
    auto walk = [&](auto eight) {
      const bool two = a.sub == 2;
      const int stages = a.stages;
      const uint32_t stage = a.stage >> 4;
      int st = 0, n = 0;
      uint32_t par = 0, at = 0;
      for (int i = first; i < a.tiles; i = next(i, ++n)) {
        const MmProduct& p = product_of<kMode>(a, tile_of<kMode>(a, i));
        const bool a_mn = kMode == MM_GRAD && p.a_mn, b_mn = kMode == MM_GRAD && p.b_mn;
        const uint32_t d = (n & 1) * kTile, idesc = mm_instr(kTile, p.tile, a.format, a_mn, b_mn);
        const uint32_t a_step = a_mn ? 128 : 2, b_step = b_mn ? 128 : 2;
        const uint32_t b_block = p.tile / 2 * kMmBlock;
        const uint64_t a_desc = smem_desc(smem, a_mn ? kHalf / 2 : 16, 1024), b_desc = smem_desc(smem + a.sub * kHalf, b_mn ? kHalf / 2 : 16, 1024);
        int steps = two ? (p.blocks[0] + 1) / 2 : p.blocks[0];
        if (kMode == MM_GRAD)
#pragma unroll
          for (int part = 1; part < kParts; ++part) steps += two ? (p.blocks[part] + 1) / 2 : p.blocks[part];
        if (!mm_wait(&bars.sum_empty[n & 1], (n >> 1 & 1) ^ 1, a.status)) return;
        fence_after();
        for (int k = 0; k < steps; ++k) {
          if (!mm_wait(&bars.full[st], par, a.status)) return;
          fence_after();
          if (one) {
            const uint64_t ad = a_desc + at, bd = b_desc + at;
#pragma unroll
            for (int j = 0; j < kMmBlock / 32; ++j) mma_pair<decltype(eight)::value>(d, ad + j * a_step, bd + j * b_step, idesc, k > 0 || j > 0);
            if (two) {
#pragma unroll
              for (int j = 0; j < kMmBlock / 32; ++j)
                mma_pair<decltype(eight)::value>(d, ad + ((kHalf >> 4) + j * a_step), bd + ((b_block >> 4) + j * b_step), idesc, true);
            }
            commit_pair(&bars.empty[st]);
          }
          at += stage;
          if (++st == stages) st = 0, par ^= 1, at = 0;
        }
        if (one) commit_pair(&bars.sum_full[n & 1]);
      }
    };
    if ((kMode == MM_LINEAR || kMode == MM_GATED) && a.eight)
      walk(std::true_type());
    else
      walk(std::false_type());
  } else if (w >= 4) {
    // ---------------------------------------------------------------- results, a row a thread, 32 columns at a time (16 with two
    // results each: registers). Between threads and memory they pass through shared memory, so that a warp's access covers
    // whole sectors of 8 rows, not 16 bytes of 32 (4096 rows of 1024 8-bit terms over 8192 columns, with a residual: 89 us)
    constexpr bool kBack = kMode == MM_BACK || kMode == MM_BACK_TWO;
    constexpr int kCols = kBack ? 16 : 32, kPieces = kCols / 8;
    constexpr bool kScaled = kMode == MM_LINEAR || kMode == MM_GATED;  // 8-bit operands, bias
    const uint32_t lanes = (uint32_t)(w & 3) << 21;
    const int id = threadIdx.x - 128, half = id >> 7;
    uint4* pass = bars.pass[w - 4];
    bool ok = true;  // (a warp whose wait ran out keeps coming to the barriers of the eight)
    // the 16-byte piece `piece` of row `r` there
    auto at_piece = [](int r, int piece) { return 4 * r + (piece ^ (r >> 1 & 3)); };
    // What a tile's columns share and its rows' own factors, asked for a tile ahead.
    struct Ahead {
      float scale = 0.f, x_scale = 1.f;
      uint16_t bias = 0;
    };
    auto look = [&](const Tile& t) {
      Ahead v;
      const MmProduct& p = product_of<kMode>(a, t);
      const MmEpilogue& e = p.e;
      const int width = one_sum(kMode) ? p.tile : p.tile / 2;
      if (kScaled && (e.x_scale || e.bias)) {
        const bool first_w = one_sum(kMode) || id < width;
        const int col = t.n0 + (first_w ? id : id - width);
        const bool in = id < p.tile && col < e.cols;
        if (in && e.x_scale) v.scale = e.w_scale[first_w ? 0 : 1][col];
        if (in && e.bias) v.bias = static_cast<const uint16_t*>(e.bias)[col];
        const long long m = t.m0 + rank * 128 + (w & 3) * 32 + lane;
        if (e.x_scale && m < e.rows) v.x_scale = e.x_scale[m];
      }
      // (what is added comes from memory: where a tile's sum takes no longer than its end it comes too late, so into the L2, lines of 128
      // bytes, two threads a row)
      if (kMode != MM_GRAD && e.in && p.blocks[0] <= 16) {
        const long long m = t.m0 + rank * 128 + (id >> 1);
        if (m < e.rows)
          for (int c = 64 * (id & 1); c < width && t.n0 + c < e.cols; c += 128)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const uint16_t*>(e.in) + m * e.in_stride + t.n0 + c));
      }
      return v;
    };
    int n = 0;
    Tile t{};
    Ahead own;
    if (first < a.tiles) t = tile_of<kMode>(a, first), own = look(t);
    for (int i = first; i < a.tiles;) {
      const Tile here = t;
      const MmProduct& p = product_of<kMode>(a, here);
      const MmEpilogue& e = p.e;
      const long long m0 = here.m0 + rank * 128 + (w & 3) * 32;
      const int width = one_sum(kMode) ? p.tile : p.tile / 2;  // results of a row
      const bool adds = kMode != MM_GRAD && e.in;
      uint4 added[kPieces];
      // (where all 32 rows and a chunk's columns are inside, its accesses go out together: one by one 434 cycles for four stores)
      const bool rows_in = m0 + 32 <= e.rows;
      const int r_in = lane / kPieces, c_in = 8 * (lane % kPieces);
      auto ask = [&](int c) {
        const int col = here.n0 + kCols * c + c_in;
        if (rows_in && here.n0 + kCols * (c + 1) <= e.cols && kCols * c < width) {
          const uint16_t* from = static_cast<const uint16_t*>(e.in) + (m0 + r_in) * e.in_stride + col;
#pragma unroll
          for (int g = 0; g < kPieces; ++g) added[g] = *reinterpret_cast<const uint4*>(from + g * (32 / kPieces) * e.in_stride);
        } else {
#pragma unroll
          for (int g = 0; g < kPieces; ++g) {
            const int r = g * (32 / kPieces) + r_in;
            added[g] = m0 + r < e.rows && col < e.cols && kCols * c < width ? load8(e.in, (m0 + r) * e.in_stride + col, e.cols - col) : make_uint4(0, 0, 0, 0);
          }
        }
      };
      if (adds) ask(half);
      if (kScaled && (e.x_scale || e.bias)) {
        asm volatile("bar.sync 1, 256;" ::: "memory");  // (the tile before has been finished with the old ones)
        bars.scale[id] = own.scale, bars.bias[id] = own.bias;
        asm volatile("bar.sync 1, 256;" ::: "memory");
      }
      const MmScale xs = mm_scale(own.x_scale);
      const int then = next(i, n + 1);
      if (then < a.tiles) t = tile_of<kMode>(a, then), own = look(t);
      const int k = n++;
      i = then;
      ok = ok && mm_wait(&bars.sum_full[k & 1], k >> 1 & 1, a.status);
      if (!ok) continue;
      fence_after();
      const uint32_t at = tmem + lanes + (k & 1) * kTile;
      mm_with_act(kMode == MM_GRAD ? FS_ACT_NONE : e.act, [&](auto act) {
        constexpr int kAct = decltype(act)::value;
#pragma unroll 1
        for (int c = half; kCols * c < width; c += 2) {
          const int n0 = here.n0 + kCols * c;
          if (n0 >= e.cols) break;
          __syncwarp();
          uint32_t z[kCols], u[kCols];
          tmem_ld(z, at + kCols * c);
          if (!one_sum(kMode)) tmem_ld(u, at + width + kCols * c);
          if (adds) {
#pragma unroll
            for (int g = 0; g < kPieces; ++g) pass[at_piece(g * (32 / kPieces) + lane / kPieces, lane % kPieces)] = added[g];
            ask(c + 2);
            __syncwarp();
          }
          wait_ld();
          uint4 y[4];  // (of a backward pass dg, then du)
          [[maybe_unused]] uint4 left[kMode == MM_BACK_TWO ? 4 : 1];  // what their rounding left
#pragma unroll
          for (int g = 0; g < kPieces; ++g) {
            const int in_tile = kCols * c + 8 * g;
            float v[8], s[8], second[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(z[8 * g + j]), second[j] = one_sum(kMode) ? 0.f : __uint_as_float(u[8 * g + j]);
            if (kScaled && e.x_scale) {
              floats8(s, bars.scale + in_tile);
              mm_scaled(v, xs, s);
              if (kMode == MM_GATED) {
                floats8(s, bars.scale + width + in_tile);
                mm_scaled(second, xs, s);
              }
            }
            if (kMode == MM_LINEAR) {
              if (e.bias) {
                floats8<T>(s, *reinterpret_cast<const uint4*>(bars.bias + in_tile));
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += s[j];
              }
#pragma unroll
              for (int j = 0; j < 8; ++j) v[j] = mm_act<kAct>(v[j]);
              if (e.in) {
                floats8<T>(s, pass[at_piece(lane, g)]);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += s[j];
              }
            } else if (kMode == MM_GRAD) {
            } else if (kMode == MM_GATED) {
#pragma unroll
              for (int j = 0; j < 8; ++j) v[j] = mm_act<kAct>(v[j]) * second[j];
            } else {
              floats8<T>(s, pass[at_piece(lane, g)]);
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                float slope;
                const float y = mm_act_slope<kAct>(v[j], slope);
                // (dy u beyond a float's range may be brought back by the slope, or be nothing with a slope of 0)
                const float dy_u = s[j] * second[j];
                v[j] = fabsf(dy_u) <= FLT_MAX ? dy_u * slope : s[j] * slope * second[j];
                second[j] = s[j] * y;
              }
              y[kPieces + g] = pack8<T>(second);
              if constexpr (kMode == MM_BACK_TWO) left[kPieces + g] = left8<T>(second, y[kPieces + g]);
            }
            y[g] = pack8<T>(v);
            if constexpr (kMode == MM_BACK_TWO) left[g] = left8<T>(v, y[g]);
          }
          auto put = [&](uint4 (&y)[4], void* one, void* other) {
            // (after all that is read of shared memory, which a store between would hold up; where a row's own addend was)
#pragma unroll
            for (int g = 0; g < 4; ++g) pass[at_piece(lane, g)] = y[g];
            __syncwarp();
            const int piece = lane % 4, col = n0 + 8 * (piece % kPieces);
            void* const out = kBack && piece >= kPieces ? other : one;
            if (rows_in && n0 + kCols <= e.cols) {
              uint16_t* to = static_cast<uint16_t*>(out) + (m0 + lane / 4) * e.out_stride + col;
#pragma unroll
              for (int g = 0; g < 4; ++g) y[g] = pass[at_piece(8 * g + lane / 4, piece)];
#pragma unroll
              for (int g = 0; g < 4; ++g) *reinterpret_cast<uint4*>(to + 8 * g * e.out_stride) = y[g];
            } else {
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                const int r = 8 * g + lane / 4;
                if (m0 + r < e.rows && col < e.cols) store8(out, (m0 + r) * e.out_stride + col, pass[at_piece(r, piece)], e.cols - col);
              }
            }
          };
          put(y, e.out[0], e.out[1]);
          if constexpr (kMode == MM_BACK_TWO) {
            __syncwarp();
            put(left, e.out[2], e.out[3]);
          }
        }
      });
      fence_before();
      __syncwarp();
      if (lane == 0) arrive_at(cluster_addr(smem_u32(&bars.sum_empty[k & 1]), 0));
    }
  }
  __syncwarp();
  fence_before();
  cluster_all();
  fence_after();
  if (w == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

template <typename T, int kMode>
cudaError_t launch(const MmWideArgs& a, int sms, cudaStream_t s) {
  static std::atomic<uint64_t> seen{0};
  const cudaError_t limit = smem_limit_once(seen, reinterpret_cast<const void*>(k_mm_wide<T, kMode>), kSmem);
  if (limit != cudaSuccess) return limit;
  const int pairs = std::min(a.tiles, std::max(1, sms / 2));
  return launch_clusters(k_mm_wide<T, kMode>, dim3(2 * pairs), dim3(kThreads), 2, kSmem, s, a);
}

template <typename T>
cudaError_t launch_mode(const MmWideArgs& a, int mode, int sms, cudaStream_t s) {
  switch (mode) {
    case MM_LINEAR: return launch<T, MM_LINEAR>(a, sms, s);
    case MM_GATED: return launch<T, MM_GATED>(a, sms, s);
    case MM_BACK: return launch<T, MM_BACK>(a, sms, s);
    case MM_BACK_TWO: return launch<T, MM_BACK_TWO>(a, sms, s);
    default: return launch<T, MM_GRAD>(a, sms, s);
  }
}

}  // namespace

cudaError_t launch_mm_wide(MmWideArgs& a, int mode, int type, int out_type, int sms, cudaStream_t s) {
  a.eight = type == FS_E4M3;
  a.format = type == FS_KV_BF16 ? 1 : 0;
  a.tiles = 0;
  a.lead = 0;
  if (mode == MM_GRAD) {  // (dx comes in first, dW of gate and up behind it)
    const MmGradPlan p = mm_grad_plan(a.product[0].e.rows, a.product[0].e.cols, a.product[1].e.rows, sms);
    if (p.dw_first) std::swap(a.product[0], a.product[2]);
    for (int i = 0; i < a.products; ++i) a.product[i].tile = p.tile;
    a.lead = p.lead;
    a.rounds = p.rounds;
  }
  int widest = 0;
  for (int i = 0; i < a.products; ++i) widest = std::max(widest, a.product[i].tile);
  // narrow tiles take two blocks a stage: their products are done before one thread's wait, products and commit for a single block are
  // (8192 terms over tiles 128 wide 27.7 -> 26.5 us, 64 wide 26.9 -> 24.3); wider ones lose more by fewer stages (160 wide 38 -> 41.7)
  a.sub = widest <= 128 ? 2 : 1;
  a.stage = a.sub * (kHalf + widest / 2 * kMmBlock);
  a.stages = std::min(kStages, kRing / a.stage);
  for (int i = 0; i < a.products; ++i) {
    MmProduct& p = a.product[i];
    const int width = one_sum(mode) ? p.tile : p.tile / 2;
    p.row_tiles = (p.e.rows + kTile - 1) / kTile;
    p.group = kGroup * ((p.e.cols + width - 1) / width);
    p.tiles = p.row_tiles * (p.group / kGroup);
    a.tiles += p.tiles;
  }
  return out_type == FS_KV_FP16 ? launch_mode<__half>(a, mode, sms, s) : launch_mode<__nv_bfloat16>(a, mode, sms, s);
}

}  // namespace fs
