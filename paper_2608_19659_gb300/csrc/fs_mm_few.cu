// Products of few rows (decode steps): W is read once, as fast as memory gives it.
//
// A tile is w_rows rows of W (the 128 rows of a tensor-core product; with fewer, its other rows are garbage that nothing
// reads) times up to 128 tokens (its columns), so that one token costs no more than 16 of padding in shared memory and
// nothing in bandwidth. Its sum is split over the blocks of a cluster, each of which leaves its share in its
// shared memory; every block then adds up and finishes a share of the tile's results, in the order of the ranks, so
// that bits repeat. Of a gated block a tile has as many rows of gate as of up.
// One lane keeps copies on their way, one issues products, all four warps take part in the end.
// Bound by reading W.
#include <algorithm>
#include <atomic>

#include "fs_mm.cuh"

namespace fs {
namespace {

constexpr int kMaxStages = 12;
constexpr int kMaxCluster = 8;

struct FewBars {
  uint64_t full[kMaxStages], empty[kMaxStages], done;
  uint32_t tmem;
};

struct MmFewArgs {
  MmEpilogue e;
  MmFewPlan p;
  int blocks_k, eight, part_at;
  uint32_t idesc;
  uint32_t* status;
};

template <bool kEight>
__device__ __forceinline__ void mma_few(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  if constexpr (kEight)
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}

// The sum over the cluster's blocks of four floats at address a of their shared memory, in the order of the ranks.
__device__ __forceinline__ float4 cluster_sum4(uint32_t a, int cluster) {
  float4 v[kMaxCluster];
#pragma unroll
  for (int i = 0; i < kMaxCluster; ++i)
    if (i < cluster)
      asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                   : "=f"(v[i].x), "=f"(v[i].y), "=f"(v[i].z), "=f"(v[i].w)
                   : "r"(cluster_addr(a, i))
                   : "memory");
  float4 s = v[0];
#pragma unroll
  for (int i = 1; i < kMaxCluster; ++i)
    if (i < cluster) s = s + v[i];
  return s;
}

template <typename T, bool kGated>
__global__ void __launch_bounds__(128) k_mm_few(const __grid_constant__ CUtensorMap mx, const __grid_constant__ CUtensorMap mw,
                                                const __grid_constant__ CUtensorMap mu, const MmFewArgs a) {
  extern __shared__ unsigned char raw[];
  const uint32_t smem = (smem_u32(raw) + 1023) & ~1023u;
  const MmFewPlan& p = a.p;
  const int slot = (p.w_rows + p.tokens) * kMmBlock, w_bytes = p.w_rows * kMmBlock;
  FewBars& bars = *reinterpret_cast<FewBars*>(raw + (smem - smem_u32(raw)) + a.part_at);
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x % p.cluster, tile = blockIdx.x / p.cluster;
  const int width = kGated ? p.w_rows / 2 : p.w_rows;  // columns of y a tile
  const int n0 = tile * width, t0 = blockIdx.y * p.tokens;
  const int k0 = (int)((long long)a.blocks_k * rank / p.cluster), k1 = (int)((long long)a.blocks_k * (rank + 1) / p.cluster);
  uint32_t cols = 32;
  while (cols < (uint32_t)p.tokens) cols *= 2;

  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.stages; ++i) mbar_init(&bars.full[i], 1), mbar_init(&bars.empty[i], 1);
    mbar_init(&bars.done, 1);
  }
  if (w == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars.tmem)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  pdl_wait();
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = bars.tmem;

  // (whole warps, with values that are the same in every lane; one lane, always the same, issues)
  if (w == 0) {
    // ---------------------------------------------------------------- copies
    const bool one = elect_one();
    if (one) fence_proxy_async_all();
    const int step = a.eight ? kMmBlock : kMmBlock / 2;
    int st = 0, k = k0;
    uint32_t par = 1;
    for (; k < k1; ++k) {
      if (!__all_sync(~0u, mm_wait(&bars.empty[st], par, a.status))) break;
      if (one) {
        const uint32_t at = smem + st * slot;
        mbar_expect_tx(&bars.full[st], slot);
        tma_rows(at, &mw, k * step, n0, &bars.full[st]);
        if (kGated) tma_rows(at + w_bytes / 2, &mu, k * step, n0, &bars.full[st]);
        tma_rows(at + w_bytes, &mx, k * step, t0, &bars.full[st]);
      }
      if (++st == p.stages) st = 0, par ^= 1;
    }
    if (k < k1)  // a wait ran out: the copies under way first (with the same limit)
      for (int j = max(k0, k - p.stages); j < k; ++j) mbar_wait(&bars.full[(j - k0) % p.stages], ((j - k0) / p.stages) & 1, kWaitLimitNs);
  } else if (w == 1) {
    // ---------------------------------------------------------------- products
    const bool one = elect_one();
    const uint32_t d = __shfl_sync(~0u, tmem, 0);
    auto walk = [&](auto eight) {
      int st = 0;
      uint32_t par = 0;
      for (int k = k0; k < k1; ++k) {
        if (!__all_sync(~0u, mm_wait(&bars.full[st], par, a.status))) break;
        fence_after();
        if (one) {
          const uint32_t at = smem + st * slot;
          const uint64_t wd = smem_desc(at, 16, 1024), xd = smem_desc(at + w_bytes, 16, 1024);
#pragma unroll
          for (int i = 0; i < kMmBlock / 32; ++i) mma_few<decltype(eight)::value>(d, wd + 2 * i, xd + 2 * i, a.idesc, k > k0 || i > 0);
          commit(&bars.empty[st]);
        }
        if (++st == p.stages) st = 0, par ^= 1;
      }
      if (one) commit(&bars.done);
    };
    if (a.eight)
      walk(std::true_type());
    else
      walk(std::false_type());
  }
  __syncwarp();
  const bool ok = mm_wait(&bars.done, 0, a.status);
  fence_after();

  // ---------------------------------------------------------------- this block's share of the sums, [token][row of W]
  const int ld = p.w_rows + 4;
  if (32 * w < p.w_rows && ok) {
    const uint32_t to = smem + (32 * w + lane) * 4;
    for (int c = 0; c < p.tokens; c += 16) {
      uint32_t x[16];
      tmem_ld16(x, tmem + ((uint32_t)(32 * w) << 16) + c);
      wait_ld();
#pragma unroll
      for (int i = 0; i < 16; ++i) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + (c + i) * ld * 4), "r"(x[i]) : "memory");
    }
  }
  fence_before();
  if (p.cluster > 1)
    cluster_all();
  else
    __syncthreads();
  fence_after();
  if (w == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols));

  // ---------------------------------------------------------------- results, four neighbours of a row at a time
  const MmEpilogue& e = a.e;
  const int quads = width / 4, items = min(p.tokens, e.rows - t0) * quads;
  mm_with_act(e.act, [&](auto act) {
    constexpr int kAct = decltype(act)::value;
    for (int i = rank * 128 + threadIdx.x; i < items; i += p.cluster * 128) {
      const int t = i / quads, q = 4 * (i % quads), n = n0 + q, left = e.cols - n;
      const long long m = t0 + t;
      if (left <= 0) continue;
      const uint32_t at = smem + (t * ld + q) * 4;
      float4 z = cluster_sum4(at, p.cluster), u = z;
      if (kGated) u = cluster_sum4(at + width * 4, p.cluster);
      if (e.x_scale) {
        const float xs = e.x_scale[m];
        z = z * xs * mm_load4(e.w_scale[0] + n, left);
        if (kGated) u = u * xs * mm_load4(e.w_scale[1] + n, left);
      }
      if (!kGated && e.bias) z = z + mm_load4(static_cast<const T*>(e.bias) + n, left);
      z = make_float4(mm_act<kAct>(z.x), mm_act<kAct>(z.y), mm_act<kAct>(z.z), mm_act<kAct>(z.w));
      if (kGated) z = z * u;
      if (!kGated && e.in) z = z + mm_load4(static_cast<const T*>(e.in) + m * e.in_stride + n, left);
      mm_store4(static_cast<T*>(e.out[0]) + m * e.out_stride + n, z, left);
    }
  });
  if (p.cluster > 1) cluster_all();  // no block leaves while another reads its shared memory
}

template <typename T, bool kGated>
cudaError_t launch(const CUtensorMap& x, const CUtensorMap& w, const CUtensorMap& u, const MmFewArgs& a, cudaStream_t s) {
  static std::atomic<uint64_t> seen{0};
  const cudaError_t limit = smem_limit_once(seen, reinterpret_cast<const void*>(k_mm_few<T, kGated>), 227 * 1024);
  if (limit != cudaSuccess) return limit;
  return launch_clusters(k_mm_few<T, kGated>, dim3(a.p.w_tiles * a.p.cluster, a.p.token_tiles), dim3(128), a.p.cluster, a.p.smem, s, x, w, u, a);
}

int part_at(const MmFewPlan& p) {
  const int slot = (p.w_rows + p.tokens) * kMmBlock;
  // (the last stage's products read 128 rows, whatever a tile has)
  const int ring = std::max(p.stages * slot, (p.stages - 1) * slot + 128 * kMmBlock);
  return std::max(ring, (p.w_rows + 4) * p.tokens * 4);
}

}  // namespace

MmFewPlan mm_few_plan(int rows, int cols, int blocks_k, bool gated, int sms) {
  MmFewPlan p{};
  p.token_tiles = (rows + 127) / 128;
  p.tokens = ((rows + p.token_tiles - 1) / p.token_tiles + 15) / 16 * 16;
  for (p.w_rows = 128;; p.w_rows /= 2) {
    const int width = gated ? p.w_rows / 2 : p.w_rows;
    p.w_tiles = (cols + width - 1) / width;
    const long long tiles = (long long)p.w_tiles * p.token_tiles;
    p.cluster = (int)std::clamp<long long>(2 * sms / tiles, 1, std::min(kMaxCluster, blocks_k));
    if (tiles * p.cluster >= sms || p.w_rows == 32) break;
  }
  const int slot = (p.w_rows + p.tokens) * kMmBlock, depth = (blocks_k + p.cluster - 1) / p.cluster;
  // two blocks an SM; and shared memory in proportion to the tensor memory, so that blocks that are resident
  // together never wait for each other's
  p.stages = std::clamp(108 * 1024 / slot, 2, std::min(kMaxStages, std::max(2, depth)));
  int columns = 32;
  while (columns < p.tokens) columns *= 2;
  p.smem = std::max<size_t>(1024 + part_at(p) + sizeof(FewBars), columns * 456);
  return p;
}

cudaError_t launch_mm_few(const CUtensorMap& x, const CUtensorMap& w, const CUtensorMap* up, const MmEpilogue& e, const MmFewPlan& p,
                          int blocks_k, int type, int out_type, uint32_t* status, cudaStream_t s) {
  const MmFewArgs a{e, p, blocks_k, type == FS_E4M3, part_at(p), mm_instr(128, p.tokens, type == FS_KV_BF16 ? 1 : 0), status};
  const bool h = out_type == FS_KV_FP16;
  if (up) return h ? launch<__half, true>(x, w, *up, a, s) : launch<__nv_bfloat16, true>(x, w, *up, a, s);
  return h ? launch<__half, false>(x, w, w, a, s) : launch<__nv_bfloat16, false>(x, w, w, a, s);
}

}  // namespace fs
