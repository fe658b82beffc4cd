// Products of few rows (decode steps): W is read once, as fast as memory gives it.
//
// A tile is w_rows rows of W (the 128 rows of a tensor-core product; with fewer, its other rows are garbage that nothing
// reads) times up to 128 tokens (its columns), so that one token costs no more than 16 of padding in shared memory and
// nothing in bandwidth. Its sum is split over the blocks of a cluster. Each of them finishes some of the tile's tokens: the
// others store their sums of those in its shared memory, and after the cluster's one barrier it adds them up, in the order of
// the ranks, so that bits repeat. Of a gated block a tile has as many rows of gate as of up.
// One warp keeps copies on their way, one issues products, all eight take part in the end.
// Tensor memory is asked for only when the kernels ahead have ended (one of them may still ask for all of it), and given back
// before the block waits for its cluster: no block that holds some waits for another.
// Bound by reading W where it is long: 64 rows of 8192 8-bit over 10240 18.6 us, the sums complete after 13.6 (6.2 TB/s), 2.2 for the
// exchange, 1.2 for the results; 8 rows of 8192 8-bit over 2 x 14336 gated 37.5 (6.3 TB/s). One row of 128 terms over 64 columns: 2.4 us,
// all latency.
#include <algorithm>
#include <atomic>

#include "fs_mm.cuh"

namespace fs {
namespace {

constexpr int kMaxStages = kFewStages, kMaxCluster = kFewCluster;
constexpr int kThreads = 256;

struct FewBars {
  uint64_t full[kMaxStages], empty[kMaxStages], done;
  uint32_t tmem;
  float x_scale[128];  // of the tokens that this block finishes
};
// Two blocks an SM: a plan's ring and sums of 111 KB, what the ring begins on, these, and the 1 KB that the system keeps.
static_assert(2 * (111 * 1024 + 1024 + sizeof(FewBars) + 1024) <= 228 * 1024, "half an SM's shared memory");

struct MmFewArgs {
  MmEpilogue e;
  MmFewPlan p;
  int blocks_k, eight, bars_at, sums_at;
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

__device__ __forceinline__ void st_cluster(uint32_t a, uint32_t x) {
  asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(a), "r"(x) : "memory");
}

// The sum of four floats of every block of the cluster, `step` bytes apart in this one's shared memory, in the order of the ranks.
__device__ __forceinline__ float4 sum4(uint32_t a, int step, int cluster) {
  float4 v[kMaxCluster];
#pragma unroll
  for (int i = 0; i < kMaxCluster; ++i)
    if (i < cluster) asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[i].x), "=f"(v[i].y), "=f"(v[i].z), "=f"(v[i].w) : "r"(a + i * step));
  float4 s = v[0];
#pragma unroll
  for (int i = 1; i < kMaxCluster; ++i)
    if (i < cluster) s = s + v[i];
  return s;
}

template <typename T, bool kGated>
__global__ void __launch_bounds__(kThreads, 2) k_mm_few(const __grid_constant__ CUtensorMap mx, const __grid_constant__ CUtensorMap mw,
                                                const __grid_constant__ CUtensorMap mu, const MmFewArgs a) {
  extern __shared__ unsigned char raw[];
  const uint32_t smem = (smem_u32(raw) + 1023) & ~1023u;
  const MmFewPlan& p = a.p;
  const int slot = (p.w_rows + p.tokens) * kMmBlock, w_bytes = p.w_rows * kMmBlock;
  FewBars& bars = *reinterpret_cast<FewBars*>(raw + (smem - smem_u32(raw)) + a.bars_at);
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
  __syncthreads();
  if (p.cluster > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // (this block has started)
  pdl_wait();
  __syncwarp();

  // What this thread's four columns of results share, asked for while the sums are made. Block `o` of the cluster finishes the
  // tokens [o share, (o + 1) share) of the tile, each kThreads / quads-th of them (kThreads is a multiple of quads) by this thread.
  const MmEpilogue& e = a.e;
  const int quads = width / 4, valid = min(p.tokens, e.rows - t0), share = tokens_each(valid, p.cluster);
  const int first = rank * share, mine = max(0, min(valid - first, share));
  const int n = n0 + 4 * (threadIdx.x % quads), left = e.cols - n, t_step = kThreads / quads;
  float4 scale0{}, scale1{};
  uint2 bias{};
  float own_scale = 1.f;  // (by the last four warps: the first two would wait for it before they copy and issue)
  if (const int i = (int)threadIdx.x - 128; e.x_scale && i >= 0 && i < mine) bars.x_scale[i] = own_scale = e.x_scale[t0 + first + i];
  if (left > 0 && mine > 0) {
    if (e.x_scale) {
      scale0 = mm_load4(e.w_scale[0] + n, left);
      if (kGated) scale1 = mm_load4(e.w_scale[1] + n, left);
    }
    if (!kGated && e.bias) bias = mm_raw4(static_cast<const uint16_t*>(e.bias) + n, left);
  }

  // (whole warps, with values that are the same in every lane; one lane, always the same, issues)
  bool ok = true;  // (of the warp: none of its waits ran out)
  if (w == 0) {
    // ---------------------------------------------------------------- copies
    const bool one = elect_one();
    if (one) fence_proxy_async_all();
    const int step = a.eight ? kMmBlock : kMmBlock / 2;
    int st = 0, k = k0;
    uint32_t par = 1;
    for (; k < k1; ++k) {
      if (!mm_wait(&bars.empty[st], par, a.status)) break;
      if (one) {
        const uint32_t at = smem + st * slot;
        mbar_expect_tx(&bars.full[st], slot);
        tma_rows(at, &mw, k * step, n0, &bars.full[st]);
        if (kGated) tma_rows(at + w_bytes / 2, &mu, k * step, n0, &bars.full[st]);
        tma_rows(at + w_bytes, &mx, k * step, t0, &bars.full[st]);
      }
      if (++st == p.stages) st = 0, par ^= 1;
    }
    ok = k == k1;
    if (!ok)  // a wait ran out: the copies under way first (with the same limit)
      for (int j = max(k0, k - p.stages); j < k; ++j) mbar_wait(&bars.full[(j - k0) % p.stages], ((j - k0) / p.stages) & 1, kWaitLimitNs);
  } else if (w == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars.tmem)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    fence_before();
    asm volatile("bar.sync 1, 64;" ::: "memory");
  } else if (w == 1) {
    // ---------------------------------------------------------------- products
    asm volatile("bar.sync 1, 64;" ::: "memory");
    fence_after();
    const bool one = elect_one();
    const uint32_t d = __shfl_sync(~0u, bars.tmem, 0);
    auto walk = [&](auto eight) {
      int st = 0;
      uint32_t par = 0;
      for (int k = k0; k < k1; ++k) {
        ok = mm_wait(&bars.full[st], par, a.status);
        if (!ok) break;
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
  ok = mm_wait(&bars.done, 0, a.status) && ok;
  fence_after();
  const uint32_t tmem = bars.tmem;  // (warp 1 has waited for it)

  // ---------------------------------------------------------------- sums to where they are added up, [rank][token][row of W]
  const int ld = 4 * p.w_rows;
  const uint32_t sums = smem + a.sums_at;
  __syncwarp();
  if (p.cluster > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // (all of them have started)
  const int group = 32 * (w & 3);  // rows of W that this warp reaches; of two such warps one takes every second eight tokens
  if (group < p.w_rows && ok) {
    const uint32_t to = sums + rank * share * ld + (group + lane) * 4, from = tmem + ((uint32_t)group << 16);
    if (valid < 8) {  // all of them the first block's
      if (w < 4) {
        uint32_t x[8];
        tmem_ld8(x, from);
        wait_ld();
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < valid) st_cluster(cluster_addr(to + i * ld, 0), x[i]);
      }
    } else {
      for (int o = 0; o * share < valid; ++o) {
        const uint32_t there = cluster_addr(to, o);
        for (int c = 8 * (w >> 2); c < share && o * share + c < valid; c += 16) {
          uint32_t x[8];
          tmem_ld8(x, from + o * share + c);
          wait_ld();
          if (o == rank) {  // (its own by the short way)
#pragma unroll
            for (int i = 0; i < 8; ++i) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + (c + i) * ld), "r"(x[i]) : "memory");
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) st_cluster(there + (c + i) * ld, x[i]);
          }
        }
      }
    }
  }
  // what a token adds, a token ahead: the first while the sums are on their way
  int t = threadIdx.x / quads;
  auto ask = [&](int ti) {
    return !kGated && e.in && ti < mine && left > 0
               ? mm_raw4(static_cast<const uint16_t*>(e.in) + (long long)(t0 + first + ti) * e.in_stride + n, left)
               : uint2{};
  };
  uint2 extra = ask(t);
  __syncwarp();
  fence_before();
  // (rare: a token's scale is far from 1, or a wait ran out)
  const bool far = __syncthreads_or(!ok || mm_scale(own_scale).far != 1.f), all = !far || __syncthreads_and(ok);
  fence_after();
  if (w == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols));
  __syncwarp();
  if (p.cluster > 1) cluster_all();  // (the last that any block does with another's shared memory)

  // ---------------------------------------------------------------- results, four neighbours of a row at a time
  if (left <= 0 || !all) return;  // (a block whose wait ran out has no sums)
  auto finish = [&](auto act, auto scales_far) {
    constexpr int kAct = decltype(act)::value;
#pragma unroll 1
    for (; t < mine; t += t_step) {  // (a small loop: its code is fetched once, while nothing else goes on)
      const uint2 own = extra;
      extra = ask(t + t_step);
      const uint32_t at = sums + t * ld + 16 * (threadIdx.x % quads);
      float4 z = sum4(at, share * ld, p.cluster), u = z;
      if (kGated) u = sum4(at + width * 4, share * ld, p.cluster);
      if (e.x_scale) {
        const float xs = bars.x_scale[t];
        if constexpr (decltype(scales_far)::value) {
          z = mm_scaled(z, mm_scale(xs), scale0);
          if (kGated) u = mm_scaled(u, mm_scale(xs), scale1);
        } else {
          z = z * xs * scale0;
          if (kGated) u = u * xs * scale1;
        }
      }
      if (!kGated) z = z + mm_floats4<T>(bias);
      z = make_float4(mm_act<kAct>(z.x), mm_act<kAct>(z.y), mm_act<kAct>(z.z), mm_act<kAct>(z.w));
      z = kGated ? z * u : z + mm_floats4<T>(own);
      mm_store4(static_cast<T*>(e.out[0]) + (t0 + first + t) * e.out_stride + n, z, left);
    }
  };
  // (a loop of its own for scales far from 1, after the others)
  if (!far)
    mm_with_act(e.act, [&](auto act) { finish(act, std::false_type()); });
  else
    mm_with_act(e.act, [&](auto act) { finish(act, std::true_type()); });
}

template <typename T, bool kGated>
cudaError_t launch(const CUtensorMap& x, const CUtensorMap& w, const CUtensorMap& u, const MmFewArgs& a, cudaStream_t s) {
  static std::atomic<uint64_t> seen{0};
  const cudaError_t limit = smem_limit_once(seen, reinterpret_cast<const void*>(k_mm_few<T, kGated>), 227 * 1024);
  if (limit != cudaSuccess) return limit;
  return launch_clusters(k_mm_few<T, kGated>, dim3(a.p.w_tiles * a.p.cluster, a.p.token_tiles), dim3(kThreads), a.p.cluster, 1024 + a.bars_at + sizeof(FewBars), s, x, w, u, a);
}

}  // namespace

cudaError_t launch_mm_few(const CUtensorMap& x, const CUtensorMap& w, const CUtensorMap* up, const MmEpilogue& e, const MmFewPlan& p,
                          int blocks_k, int type, int out_type, uint32_t* status, cudaStream_t s) {
  const MmFewArgs a{e, p, blocks_k, type == FS_E4M3, bars_at(p, e.rows), sums_at(p), mm_instr(128, p.tokens, type == FS_KV_BF16 ? 1 : 0), status};
  const bool h = out_type == FS_KV_FP16;
  if (up) return h ? launch<__half, true>(x, w, *up, a, s) : launch<__nv_bfloat16, true>(x, w, *up, a, s);
  return h ? launch<__half, false>(x, w, w, a, s) : launch<__nv_bfloat16, false>(x, w, w, a, s);
}

}  // namespace fs
