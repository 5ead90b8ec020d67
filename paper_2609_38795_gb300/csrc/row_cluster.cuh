// A row of logits held in the registers of a thread-block cluster.
//
// A row (up to 1 MB) is read from memory once and stays on chip for all that an operator does with it:
// C blocks of T threads hold kPacks 16-byte packs each.  Warps own consecutive stretches of the
// row, in the order (block, warp, pack, lane), so that "first" and "running sum" follow from records per
// warp, and every warp-wide access is 512 consecutive bytes.
//
// Rows need not be 16-byte aligned: packs are counted from the 16-byte boundary at or below the row's
// first element, and the elements of the first and the last pack that are not the row's read as -inf.
#pragma once

#include <algorithm>
#include <mutex>
#include <type_traits>

#include "launch.h"
#include "row_reduce.cuh"

namespace alr {

constexpr int kRowThreadsMost = 480;   // and a warp that fetches: 512, two blocks of 64 registers an SM
constexpr int kRowWarpsMost = kRowThreadsMost / 32;
constexpr int kRowClusterMost = 8;

// Launch shape: threads T of a block, blocks C of a cluster, packs a thread holds.
struct RowShape {
  int threads, cluster, packs;
};

constexpr int kRowPackChoices[] = {2, 5, 10, 18};

// Few rows: as many blocks as give every SM one, and few packs a thread (the row's latency is what
// counts).  Many rows: the fewest blocks that hold the row at 10 packs a thread, two or more of which share
// an SM, so that one's transfers overlap the other's arithmetic (loss and gradient of 2048 x 151936 bf16 logits,
// 40 % of the rows masked, in an earlier form of the kernel: 214 us in clusters of 4; 297 in clusters of 8 half
// as large, 241 in clusters of 2 twice as large, one block to an SM).  18 packs a thread are for fp32 rows of more than 150 K tokens,
// which 8 blocks hold no other way.
// `least`: threads that a block should have if the row is long enough.
inline RowShape row_shape(long long N, int V, int elem_bytes, int sms, int least = 64) {
  const int per = 16 / elem_bytes;
  const int need = (V + per - 1) / per + 1;   // one more for a row that starts inside a pack
  const auto fits = [need](int c, int packs) {
    return (need + c * packs - 1) / (c * packs) <= kRowThreadsMost;
  };
  RowShape s{0, 1, 10};
  while (s.cluster < kRowClusterMost && !fits(s.cluster, 10)) s.cluster *= 2;
  while (s.cluster < kRowClusterMost && N * s.cluster < sms && need > s.cluster * 512) s.cluster *= 2;
  if (!fits(s.cluster, 10)) {
    s.packs = 18;
  } else if (N * s.cluster <= 2 * sms) {
    for (int p : kRowPackChoices)
      if (fits(s.cluster, p)) {
        s.packs = p;
        break;
      }
  }
  const auto threads = [&] { return (need + s.cluster * s.packs - 1) / (s.cluster * s.packs); };
  for (int p : {5, 2})
    if (s.packs > p && threads() < least && fits(s.cluster, p)) s.packs = p;
  const int t = threads();
  s.threads = std::max(64, (t + 31) / 32 * 32);
  return s;
}

// Clusters of a kernel that the device holds at once (0: none); asked for once per kernel and shape.
inline int resident_clusters(const void* kern, const cudaLaunchConfig_t& cfg, int cluster) {
  struct Known {
    const void* kern;
    int dev, threads, cluster;
    size_t smem;
    int n;
  };
  static Known table[256];
  static int used = 0;
  static std::mutex mu;
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  const int threads = int(cfg.blockDim.x);
  const std::lock_guard<std::mutex> lock(mu);
  for (int i = 0; i < used; ++i)
    if (table[i].kern == kern && table[i].dev == dev && table[i].threads == threads &&
        table[i].cluster == cluster && table[i].smem == cfg.dynamicSmemBytes)
      return table[i].n;
  if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) {
    (void)cudaGetLastError();   // a shape the device cannot place: not an error of the call
    n = 0;
  }
  if (used < 256) table[used++] = {kern, dev, threads, cluster, cfg.dynamicSmemBytes, n};
  return n;
}

// Calls f(std::integral_constant<int, packs>).
template <typename F>
cudaError_t with_packs(int packs, F f) {
  switch (packs) {
    case 2: return f(std::integral_constant<int, 2>{});
    case 5: return f(std::integral_constant<int, 5>{});
    case 10: return f(std::integral_constant<int, 10>{});
    default: return f(std::integral_constant<int, 18>{});
  }
}

// Launches a cluster for each row.
template <typename... KArgs, typename... Args>
cudaError_t launch_row_each(const RowShape& shape, long long N, void (*kern)(KArgs...),
                            cudaStream_t s, const Args&... args) {
  cudaLaunchAttribute attr[2] = {pdl_attribute(), {}};
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = unsigned(shape.cluster);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(N * shape.cluster));
  cfg.blockDim = dim3(unsigned(shape.threads));
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

// Launches clusters that take the N rows in turn: as many as there are rows, or as the device holds.
template <typename... KArgs, typename... Args>
cudaError_t launch_row_clusters(const RowShape& shape, int threads, size_t smem, long long N, int sms,
                                void (*kern)(KArgs...), cudaStream_t s, const Args&... args) {
  cudaError_t e =
      cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[2] = {pdl_attribute(), {}};
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = unsigned(shape.cluster);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(shape.cluster));
  cfg.blockDim = dim3(unsigned(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  long long clusters = N;
  if (N * shape.cluster > sms) {
    const int most = resident_clusters(reinterpret_cast<const void*>(kern), cfg, shape.cluster);
    if (most > 0) clusters = std::min<long long>(N, most);
  }
  cfg.gridDim = dim3(unsigned(std::min<long long>(clusters, 1 << 20) * shape.cluster));
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

template <typename E>
constexpr int kPerPack = 16 / int(sizeof(E));

// Where a thread's packs lie.
template <typename E, int kPacks>
struct RowPlace {
  int off;    // elements of the first pack that lie before the row
  int pack;   // this lane's pack 0; pack i is 32 i further
  int base;   // the block's first pack
  ALR_DEV RowPlace(long long row_start, int rank, int threads) {
    off = int(row_start % kPerPack<E>);
    base = rank * threads * kPacks;
    pack = base + (int(threadIdx.x) / 32) * 32 * kPacks + (int(threadIdx.x) & 31);
  }
  // First element of pack i (may be negative or past the row).
  ALR_DEV int elem(int i) const { return (pack + 32 * i) * kPerPack<E> - off; }
  // Every pack of the warp lies within the row: the same answer in all its lanes, and the warp's
  // loads and stores need no checks.
  ALR_DEV bool whole(int V) const {
    const int first = pack - int(threadIdx.x & 31);
    return first * kPerPack<E> >= off && (first + 32 * kPacks) * kPerPack<E> - off <= V;
  }
};

ALR_DEV uint32_t raw_bits(__nv_bfloat16 x) { return __bfloat16_as_ushort(x); }

template <typename E>
ALR_DEV uint4 neg_inf_pack() {
  const uint32_t w = sizeof(E) == 2 ? 0xff80ff80u : 0xff800000u;
  return make_uint4(w, w, w, w);
}

// Pack of the row's elements [v, v + kPerPack), -inf where there is none.  `row`: its first element.
template <typename E>
ALR_DEV uint4 load_pack(const E* row, int v, int V) {
  if (v >= 0 && v + kPerPack<E> <= V) return __ldcs(reinterpret_cast<const uint4*>(row + v));
  uint4 r = neg_inf_pack<E>();
  if (v >= V || v + kPerPack<E> <= 0) return r;
  uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int e = 0; e < kPerPack<E>; ++e) {
    if (v + e < 0 || v + e >= V) continue;
    if constexpr (sizeof(E) == 2) {
      const uint32_t b = raw_bits(row[v + e]);
      w[e / 2] = e & 1 ? (w[e / 2] & 0xffffu) | (b << 16) : (w[e / 2] & 0xffff0000u) | b;
    } else {
      w[e] = __float_as_uint(row[v + e]);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Element e of a pack (e known when unrolled).
template <typename E>
ALR_DEV float pack_elem(const uint4& r, int e) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
  if constexpr (sizeof(E) == 2)
    return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
  else
    return __uint_as_float(w[e]);
}

// Elements of a pack whose bit in `bits` is set become -inf.  A loop over the set bits, of which
// there are next to none: unrolled selects would be executed for every pack.
template <typename E>
ALR_DEV void mask_pack(uint4& r, uint32_t bits) {
  while (bits != 0) {
    const int e = __ffs(bits) - 1;
    bits &= bits - 1;
    const int word = sizeof(E) == 2 ? e >> 1 : e;
    const uint32_t m = sizeof(E) == 4 ? 0xffffffffu : e & 1 ? 0xffff0000u : 0xffffu;
    const uint32_t inf = (sizeof(E) == 4 ? 0xff800000u : 0xff80ff80u) & m;
    if (word == 0) r.x = (r.x & ~m) | inf;
    if (word == 1) r.y = (r.y & ~m) | inf;
    if (word == 2) r.z = (r.z & ~m) | inf;
    if (word == 3) r.w = (r.w & ~m) | inf;
  }
}

// A pair of floats into another block's (or this one's) shared memory, counted by the mbarrier there.
ALR_DEV void st_async_f2(uint32_t cluster_addr, float x, float y, uint32_t cluster_mbar) {
  asm volatile(
      "st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];" ::"r"(
          cluster_addr),
      "r"(__float_as_uint(x)), "r"(__float_as_uint(y)), "r"(cluster_mbar)
      : "memory");
}

// mbar_wait for a phase that other blocks of the cluster complete.
ALR_DEV bool mbar_wait_cluster(uint64_t* bar, uint32_t parity, const AbortFlag& ab) {
  const uint64_t t0 = global_timer_ns();
  for (uint32_t i = 1;; ++i) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(smem_u32(bar)), "r"(parity), "r"(kSuspendHintNs)
        : "memory");
    if (done) return true;
    if (i % kWaitCheckEvery == 0) {
      if (*ab.smem) return false;
      if (global_timer_ns() - t0 > kWaitLimitNs) {
        *ab.smem = 1;
        atomicExch(ab.status, kStatusTimeout);
        return false;
      }
    }
  }
}

// Consecutive bytes of global memory into shared memory (all 16-byte multiples).
ALR_DEV void bulk_load(uint32_t smem, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
          smem),
      "l"(__cvta_generic_to_global(src)), "r"(bytes), "r"(smem_u32(bar))
      : "memory");
}

// The two halves of cluster_sync.
ALR_DEV void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
// Without ordering anything: arrive early, where loads are in flight that a release would wait for.
ALR_DEV void cluster_arrive_relaxed() {
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
ALR_DEV void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

ALR_DEV void named_bar_arrive(int id, int nthreads) {
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(nthreads) : "memory");
}

}  // namespace alr
