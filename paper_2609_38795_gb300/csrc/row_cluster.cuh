// A row of logits held in the registers of a thread-block cluster.
//
// A row (up to 1 MB) is read from memory once and stays on chip for all that an operator does with it:
// C blocks of T threads hold kPacks 16-byte packs each.  Warps own consecutive stretches of the
// row, in the order (block, warp, pack, lane), so that "first" and "running sum" follow from records per
// warp, and every warp-wide load is 512 consecutive bytes.
//
// Rows need not be 16-byte aligned: packs are counted from the 16-byte boundary at or below the row's
// first element, and the elements of the first and the last pack that are not the row's read as -inf.
#pragma once

#include <type_traits>

#include "launch.h"
#include "row_reduce.cuh"

namespace alr {

constexpr int kRowThreadsMost = 512;
constexpr int kRowWarpsMost = kRowThreadsMost / 32;
constexpr int kRowClusterMost = 8;

// Launch shape: threads T of a block, blocks C of a cluster, packs a thread holds.
struct RowShape {
  int threads, cluster, packs;
};

constexpr int kRowPackChoices[] = {2, 5, 10, 18};

// Few rows: as many blocks as give every SM one, and few packs a thread (the row's latency is what
// counts).  Many rows: the fewest blocks that hold the row at 10 packs a thread, 2 to 4 blocks of 512
// threads at most to an SM, whose loads overlap the others' arithmetic.  18 packs a thread are for
// fp32 rows of more than 160 K tokens, which 8 blocks of 512 threads hold no other way.
inline RowShape row_shape(long long N, int V, int elem_bytes, int sms) {
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
  const int t = (need + s.cluster * s.packs - 1) / (s.cluster * s.packs);
  s.threads = (t + 31) / 32 * 32;
  if (s.threads < 64) s.threads = 64;
  return s;
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

// N rows, a cluster (or, of one, a block) each.
template <typename... KArgs, typename... Args>
cudaError_t launch_row_clusters(const RowShape& shape, long long N, void (*kern)(KArgs...),
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
  cfg.numAttrs = shape.cluster > 1 ? 2 : 1;
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
  ALR_DEV RowPlace(long long row_start, int rank) {
    off = int(row_start % kPerPack<E>);
    base = rank * int(blockDim.x) * kPacks;
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

// The thread's packs of a row.
template <typename E, int kPacks>
ALR_DEV void load_row(uint4 (&raw)[kPacks], const E* row, const RowPlace<E, kPacks>& at, int V) {
  if (at.whole(V)) {
    const uint4* p = reinterpret_cast<const uint4*>(row + at.elem(0));
#pragma unroll
    for (int i = 0; i < kPacks; ++i) raw[i] = __ldcs(p + 32 * i);
  } else {
#pragma unroll
    for (int i = 0; i < kPacks; ++i) raw[i] = load_pack(row, at.elem(i), V);
  }
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

// Records of the cluster's warps, written by each into its own block's shared memory; after a
// cluster_sync (one block: __syncthreads) any thread reads record i of the n = C * warps, in the
// order of the row.
ALR_DEV float2 ld_cluster_f2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
  return v;
}
ALR_DEV void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
ALR_DEV void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

}  // namespace alr
