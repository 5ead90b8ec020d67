// A teacher's top logits, and the next token of a rollout drawn from given random numbers.
//
// Both pick from a row by the order (value descending, token id ascending).  A logit that is -inf or
// NaN is no candidate.
//
// Rows.  Few rows: each in the registers of a cluster, read once (row_cluster.cuh, `Row`): the row's latency is
// what counts.  From a row per SM on: each read by one block (`StreamRow`), two blocks to an SM, no cluster
// barriers, and one block reads while the other selects; what needs a second sweep finds the row in L2.
// 768 x 151936 bf16 rows, top-k and top-p: 78 us streamed (3.0 TB/s), 164 us in clusters.
//
// Few tokens of many (top logits, top-k): the K-th largest of the largest logits that the threads hold is a
// lower bound of the row's K-th largest, and not many more than K logits reach it.  Those are sorted by the
// first block.  A streamed row takes the bound from its first packs and holds the rest against it as it
// comes by: one reading in all.
// Any number of tokens (a nucleus, a top-k past kTopMost): a histogram of counts or weights over even steps
// of the logit below the largest, in each block's shared memory and added up over the cluster, tells the
// step in which the cut falls; that step's logits are sorted as above.  A returning shared-memory atomic
// for each logit is what that costs (some 150 K cycles for 2 x 152 K logits on an SM), so only the logits of
// the upper 16 octaves have one at first.  A nucleus of trained rows: 244 us for 768 x 151936, of a random
// head's, whose bulk it takes in, 738 us.
// So many equal logits that they do not fit: a radix select over an order-preserving key.
//
// Bound by latency and instructions, not by memory: see the figures at the steps.  Sweeps over weights are
// loops of little code on purpose (each_heavy): unrolled, half of their stalls were for instructions.
#include "kernels.h"
#include "launch.h"
#include "row_cluster.cuh"

namespace alr {
namespace {

constexpr int kBins = 2048;              // of a histogram: 11 bits of a key, or steps of 1/64 octave
constexpr int kCandMost = 1024;          // candidates of a row
constexpr int kCandSort = 256;           // up to here an entry's place is counted, beyond they are sorted
constexpr int kStreamThreads = 512;      // of a block that reads a row by itself
constexpr int kSlots = 4;                // places that a warp has for its candidates without asking
constexpr int kListMost = kTopMost + 2 * kRowWarpsMost * kRowClusterMost;
constexpr int kListWarp = 256;           // a list that long is one warp's work, a longer one the block's
constexpr int kWarpsMost = kRowWarpsMost * kRowClusterMost;

// An entry: larger is earlier in the order.
ALR_DEV unsigned long long entry(uint32_t key, int v) {
  return ((unsigned long long)key << 32) | uint32_t(~v);
}
ALR_DEV uint32_t entry_key(unsigned long long e) { return uint32_t(e >> 32); }
ALR_DEV int entry_id(unsigned long long e) { return int(~uint32_t(e)); }

// What a row keeps: keys above `key`, and of the tokens with that key those up to id `last`.
struct Cut {
  uint32_t key;
  int last;
  ALR_DEV bool keeps(uint32_t k, int v) const { return k > key || (k == key && v <= last); }
};

struct Shared {
  union {
    struct {
      unsigned long long all[kCandMost];  // first block: the candidates in order
      unsigned long long w[kTopMost];     // their weights
      float list[kListMost];              // largest logits of the warps' threads
    } few;
    struct {
      uint32_t lo[kBins], hi[kBins];      // histogram: sums, and the carries out of them
      unsigned long long total[kBins];    // over the cluster
    } many;
  };
  unsigned long long cand[kCandMost];     // first block: candidates, kSlots places a warp, then more
  int count[kWarpsMost + 1];              // first block: in each warp's places; then their offsets
  uint32_t small[256];                    // histogram of the list's keys
  unsigned long long rec[kWarpsMost];     // of each warp of the cluster (or batch of a streamed row): a sum
  unsigned long long grid[8 * kStreamThreads / 32];   // of a batch's packs and warps
  float2 frec[kWarpsMost];
  float fbuf[32];
  unsigned long long lbuf[32];
  int n_more;                             // first block: candidates past the warps' places
  uint32_t digit, reach;
  unsigned long long above, found, kept;
  int kept_n;
};

ALR_DEV float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Element e of a pack, e not known to the compiler.
template <typename E>
ALR_DEV float pack_elem_at(const uint4& r, int e) {
  const int word = sizeof(E) == 2 ? e >> 1 : e;
  const uint32_t w = word == 0 ? r.x : word == 1 ? r.y : word == 2 ? r.z : r.w;
  return __uint_as_float(sizeof(E) == 4 ? w : e & 1 ? w & 0xffff0000u : w << 16);
}

ALR_DEV float pack_largest(const uint4& r, std::integral_constant<int, 2>) {
  float m = kNegInf;
#pragma unroll
  for (int e = 0; e < 8; e += 2)
    m = max3(m, pack_elem<__nv_bfloat16>(r, e), pack_elem<__nv_bfloat16>(r, e + 1));
  return m;
}
ALR_DEV float pack_largest(const uint4& r, std::integral_constant<int, 4>) {
  return max3(max3(kNegInf, pack_elem<float>(r, 0), pack_elem<float>(r, 1)), pack_elem<float>(r, 2),
              pack_elem<float>(r, 3));
}
template <typename E>
ALR_DEV float largest(const uint4& r) {
  return pack_largest(r, std::integral_constant<int, int(sizeof(E))>{});
}

// Elements of a pack that reach `least`, a bit each.  Where few do, a loop over the bits set costs the warp
// an element's instructions or two; a loop over the elements costs it all of them for one lane's one.
template <typename E>
ALR_DEV uint32_t reaching(const uint4& r, float least) {
  uint32_t bits = 0;
#pragma unroll
  for (int e = 0; e < kPerPack<E>; ++e) bits |= uint32_t(pack_elem<E>(r, e) >= least) << e;
  return bits;
}

// NaN elements of a pack become -inf.
template <typename E>
ALR_DEV void clean(uint4& r) {
  float m = kNegInf;
#pragma unroll
  for (int e = 0; e < kPerPack<E>; e += 2)
    m = max3_nan(m, pack_elem<E>(r, e), pack_elem<E>(r, e + 1));
  if (m == m) return;
  uint32_t bits = 0;
#pragma unroll
  for (int e = 0; e < kPerPack<E>; ++e) bits |= uint32_t(pack_elem<E>(r, e) != pack_elem<E>(r, e)) << e;
  mask_pack<E>(r, bits);
}

// What all threads of a row's cluster need to know.  kSolo: the cluster is one block.
template <bool kSolo>
struct RowCommon {
  int V, rank, cluster, warp, lane, n_warps;
  float most;      // largest element that the thread holds (from row_bound on)
  bool infinite;   // the row has +inf logits, which have all the mass: they read as 0, others as -inf
  Shared& sh;

  ALR_DEV RowCommon(int V_, int cluster_, Shared& s)
      : V(V_),
        rank(kSolo ? 0 : int(cluster_ctarank())),
        cluster(kSolo ? 1 : cluster_),
        warp(int(threadIdx.x) / 32),
        lane(int(threadIdx.x) & 31),
        n_warps(int(blockDim.x) / 32),
        most(kNegInf),
        infinite(false),
        sh(s) {}
  ALR_DEV int record() const { return rank * n_warps + warp; }
  ALR_DEV int records() const { return cluster * n_warps; }
  ALR_DEV void sync() const {
    if constexpr (kSolo)
      __syncthreads();
    else
      cluster_sync();
  }
  // A warp-uniform value into a slot of every block's shared memory.
  template <typename T>
  ALR_DEV void to_all(T* slot, T v) const {
    if constexpr (kSolo) {
      if (lane == 0) *slot = v;
    } else if (lane < cluster) {
      put(cluster_smem_addr(slot, lane), v);
    }
  }
  template <typename T>
  ALR_DEV void to_first(T* slot, T v) const {
    if constexpr (kSolo)
      *slot = v;
    else
      put(cluster_smem_addr(slot, 0), v);
  }
  template <typename T>
  ALR_DEV static void put(uint32_t a, T v) {
    if constexpr (sizeof(T) == 8) {
      unsigned long long b;
      memcpy(&b, &v, 8);
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(b) : "memory");
    } else {
      uint32_t b;
      memcpy(&b, &v, 4);
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a), "r"(b) : "memory");
    }
  }
  ALR_DEV int add_first(int* slot, int v) const {
    if constexpr (kSolo) return atomicAdd(slot, v);
    int r;
    asm volatile("atom.shared::cluster.add.s32 %0, [%1], %2;"
                 : "=r"(r)
                 : "r"(cluster_smem_addr(slot, 0)), "r"(v)
                 : "memory");
    return r;
  }
  ALR_DEV uint32_t from(const uint32_t* slot, int block) const {
    if constexpr (kSolo) return *slot;
    return uint32_t(ld_cluster_s32(cluster_smem_addr(slot, block)));
  }
};

template <typename E>
ALR_DEV void zero_for_infinite(uint4& r) {
  uint32_t bits = 0;
#pragma unroll
  for (int e = 0; e < kPerPack<E>; ++e) bits |= uint32_t(pack_elem<E>(r, e) != -kNegInf) << e;
  r = make_uint4(0, 0, 0, 0);
  mask_pack<E>(r, bits);
}

// The row in the registers of a cluster: each warp a stretch of it.
template <typename E_, int kPacks>
struct Row : RowCommon<false> {
  using E = E_;
  uint4 raw[kPacks];
  RowPlace<E, kPacks> at;

  ALR_DEV Row(const E* z, long long start, int V_, int cluster_, Shared& s)
      : RowCommon<false>(V_, cluster_, s), at(start, int(cluster_ctarank()), int(blockDim.x)) {
    if (at.whole(V)) {
      const uint4* p = reinterpret_cast<const uint4*>(z + at.elem(0));
#pragma unroll
      for (int i = 0; i < kPacks; ++i) raw[i] = __ldcs(p + 32 * i);
    } else {
#pragma unroll
      for (int i = 0; i < kPacks; ++i) raw[i] = load_pack(z, at.elem(i), V);
    }
    cluster_arrive_relaxed();   // ready() waits: the other blocks run, their shared memory is there
  }
  ALR_DEV void ready() const { cluster_wait(); }
  // f(pack, id of its first element) for the thread's packs, in order; every lane of the warp calls.
  template <typename F>
  ALR_DEV void each(F f) {
#pragma unroll
    for (int i = 0; i < kPacks; ++i) f(raw[i], at.elem(i));
  }
  // The same for an f of many instructions: a loop, so that the code stays in the instruction cache
  // (unrolled, the sweeps over weights stalled on it most of their time).  Only on a copy of the row,
  // which lies in local memory for it.
  template <typename F>
  ALR_DEV void each_heavy(F f) {
#pragma unroll 1
    for (int i = 0; i < kPacks; ++i) f(raw[i], at.elem(i));
  }
  template <typename F>
  ALR_DEV void each_first(F f) {   // before all others: NaN elements go
#pragma unroll
    for (int i = 0; i < kPacks; ++i) {
      clean<E>(raw[i]);
      f(raw[i], at.elem(i));
    }
  }
  // The same, packs of all lanes one after another; f returns true to stop (the same in all lanes).
  template <typename F>
  ALR_DEV void each_until(F f) {
    bool stop = false;
#pragma unroll 1
    for (int i = 0; i < kPacks && !stop; ++i) {
      uint4 r = raw[0];
#pragma unroll
      for (int j = 1; j < kPacks; ++j)
        if (j == i) r = raw[j];
      stop = f(r, at.elem(i));
    }
  }
  ALR_DEV void only_infinite() {
    infinite = true;
#pragma unroll
    for (int i = 0; i < kPacks; ++i) zero_for_infinite<E>(raw[i]);
    most = most == -kNegInf ? 0.f : kNegInf;
  }
};

// The row read anew (from the second time on, out of L2) by one block: pack j of a thread in batch b is
// (b kBatch + j) T + its number, so that however few tokens a mask leaves, many threads hold some.
template <typename E_>
struct StreamRow : RowCommon<true> {
  using E = E_;
  static constexpr int kBatch = 8;
  const E* z;
  int off, packs, batches;   // the row starts `off` elements into pack 0

  ALR_DEV StreamRow(const E* z_, long long start, int V_, Shared& s)
      : RowCommon<true>(V_, 1, s), z(z_), off(int(start % kPerPack<E>)) {
    packs = (V + off + kPerPack<E> - 1) / kPerPack<E>;
    batches = (packs + kStreamThreads * kBatch - 1) / (kStreamThreads * kBatch);
  }
  ALR_DEV void ready() const { __syncthreads(); }   // the last row's shared memory is free
  // First element of the thread's pack j in batch b.
  ALR_DEV int elem(int b, int j) const {
    return ((b * kBatch + j) * kStreamThreads + int(threadIdx.x)) * kPerPack<E> - off;
  }
  // Packs first .. first + kN of the thread, counted through the batches.
  template <int kN>
  ALR_DEV void load(uint4 (&raw)[kN], int first) const {
    const int v = elem(0, first);
    if ((first > 0 || off == 0) && elem(0, first + kN) - int(threadIdx.x) * kPerPack<E> <= V) {
      const uint4* q = reinterpret_cast<const uint4*>(z + v);
#pragma unroll
      for (int j = 0; j < kN; ++j) raw[j] = q[kStreamThreads * j];
    } else {
#pragma unroll
      for (int j = 0; j < kN; ++j) raw[j] = load_pack(z, elem(0, first + j), V);
    }
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      clean<E>(raw[j]);
      if (infinite) zero_for_infinite<E>(raw[j]);
    }
  }
  ALR_DEV uint4 load_one(int i) const {
    uint4 p = load_pack(z, elem(0, i), V);
    clean<E>(p);
    if (infinite) zero_for_infinite<E>(p);
    return p;
  }
  template <typename F>
  ALR_DEV void each(F f) {
    for (int b = 0; b < batches; ++b) {
      uint4 raw[kBatch];
      load(raw, b * kBatch);
#pragma unroll
      for (int j = 0; j < kBatch; ++j) f(raw[j], elem(b, j));
    }
  }
  // The same for an f of many instructions, with fewer copies of it.
  static constexpr int kHeavy = 2;
  template <typename F>
  ALR_DEV void each_heavy(F f) {
    const int most = (packs + kStreamThreads - 1) / kStreamThreads;   // of a thread
#pragma unroll 1
    for (int i = 0; i < most; i += 2 * kHeavy) {
      uint4 raw[2 * kHeavy];
      load(raw, i);
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int j = 0; j < kHeavy; ++j) f(raw[j], elem(0, i + h * kHeavy + j));
#pragma unroll
        for (int j = 0; j < kHeavy; ++j) raw[j] = raw[j + kHeavy];
      }
    }
  }
  template <typename F>
  ALR_DEV void each_first(F f) {
    each(f);
  }
  ALR_DEV void only_infinite() {
    infinite = true;
    most = most == -kNegInf ? 0.f : kNegInf;
  }
};

// The n-th (from 1) unit of weight f(x, id) >= 0, counted in the order of ids over the whole row: the
// id of the token that holds it, that token's weight and the sum of all weights.  n(total) gives n.
// f(x, id) is 0 for logits below `least`; f.pack and f.few sum over a pack's elements, the second one by one.
struct Found {
  int id;
  unsigned long long weight, total;
  int count;   // this thread's tokens, where f counts them
};
template <typename F>
ALR_DEV auto counted(const F& f) -> decltype(f.count) { return f.count; }
ALR_DEV int counted(...) { return 0; }
template <typename E, typename F>
struct OfPack {
  F f;
  ALR_DEV unsigned long long operator()(float x, int id) { return f(x, id); }
  ALR_DEV unsigned long long pack(const uint4& p, int id, float least) { return few(p, id, least); }
  ALR_DEV unsigned long long few(const uint4& p, int id, float least) {
    unsigned long long s = 0;
    for (uint32_t bits = reaching<E>(p, least); bits != 0; bits &= bits - 1) {
      const int e = __ffs(bits) - 1;
      s += f(pack_elem_at<E>(p, e), id + e);
    }
    return s;
  }
};

// The sum of a pack's weights; all lanes of a warp call.
template <typename E, typename F>
ALR_DEV unsigned long long sum_of_pack(F& f, const uint4& p, int id, float least) {
  const bool some = largest<E>(p) >= least;
  const int lanes = __popc(__ballot_sync(0xffffffffu, some));
  if (lanes == 0) return 0;
  if (lanes >= 8) return f.pack(p, id, least);
  return some ? f.few(p, id, least) : 0ull;
}

template <typename E, int kPacks, typename F, typename N>
ALR_DEV Found find_unit(Row<E, kPacks>& row, float least, F f, N nth) {
  Shared& sh = row.sh;
  unsigned long long s = 0;
  row.each_heavy([&](const uint4& p, int id) {
    s += sum_of_pack<E>(f, p, id, least);
  });
  s = warp_reduce(s, AddOp());
  row.to_all(&sh.rec[row.record()], s);
  row.sync();
  unsigned long long total = 0, before = 0;
  for (int i = row.lane; i < row.records(); i += 32) {
    const unsigned long long t = sh.rec[i];
    total += t;
    if (i < row.record()) before += t;
  }
  total = warp_reduce(total, AddOp());
  before = warp_reduce(before, AddOp());
  const int count = counted(f);   // of the first sweep; what the search adds is not wanted
  const unsigned long long n = nth(total);
  if (before < n && n <= before + s)   // this warp holds it
    row.each_until([&](const uint4& p, int id) {
      const unsigned long long mine = sum_of_pack<E>(f, p, id, least);
      unsigned long long incl = warp_scan(mine);
      const unsigned long long all = __shfl_sync(0xffffffffu, incl, 31);
      if (n > before + all) {
        before += all;
        return false;
      }
      unsigned long long run = before + incl - mine, w = 0;
      int at = -1;
      if (run < n && n <= run + mine)
#pragma unroll 1
        for (int e = 0; e < kPerPack<E>; ++e) {
          const unsigned long long t = f(pack_elem_at<E>(p, e), id + e);
          if (at < 0 && run < n && n <= run + t) {
            at = id + e;
            w = t;
          }
          run += t;
        }
      const int src = (__ffs(__ballot_sync(0xffffffffu, at >= 0)) - 1) & 31;
      row.to_all(&sh.found, (unsigned long long)uint32_t(__shfl_sync(0xffffffffu, at, src)));
      row.to_all(&sh.kept, __shfl_sync(0xffffffffu, w, src));
      return true;
    });
  row.sync();
  const Found r{int(uint32_t(sh.found)), sh.kept, total, count};
  row.sync();   // before `found` and `rec` are written again
  return r;
}

// A weight (up to 2^31) into its bin: 32 bits of the sum and a count of the carries.
ALR_DEV void add_bin(Shared& sh, uint32_t b, uint32_t w) {
  if (atomicAdd(&sh.many.lo[b], w) + w < w) atomicAdd(&sh.many.hi[b], 1u);
}

// many.total of all blocks from the blocks' histograms; each block adds up a share of the bins.
template <typename R>
ALR_DEV void total_bins(R& row, int bins) {
  Shared& sh = row.sh;
  const int share = (bins + row.cluster - 1) / row.cluster;
  for (int b = row.rank * share + int(threadIdx.x); b < min(bins, (row.rank + 1) * share);
       b += blockDim.x) {
    unsigned long long t = 0;
    for (int c = 0; c < row.cluster; ++c)
      t += row.from(&sh.many.lo[b], c) + ((unsigned long long)row.from(&sh.many.hi[b], c) << 32);
    for (int c = 0; c < row.cluster; ++c) {
      if (row.cluster == 1)
        sh.many.total[b] = t;
      else
        R::put(cluster_smem_addr(&sh.many.total[b], c), t);
    }
  }
  row.sync();
}

// The order of a streamed row is batch, pack, thread: sums per batch tell the batch, sums per pack and
// warp of that batch the warp.
template <typename E, typename F, typename N>
ALR_DEV Found find_unit(StreamRow<E>& row, float least, F f, N nth) {
  Shared& sh = row.sh;
  constexpr int kBatch = StreamRow<E>::kBatch, kWarps = kStreamThreads / 32;
  static_assert(262144 / kPerPack<E> / (kStreamThreads * kBatch) + 2 <= kWarpsMost, "a sum per batch");
  for (int i = threadIdx.x; i < row.batches; i += blockDim.x) sh.rec[i] = 0;
  __syncthreads();
  const auto of_pack = [&](const uint4& p, int id) {
    return sum_of_pack<E>(f, p, id, least);
  };
  const int most = (row.packs + kStreamThreads - 1) / kStreamThreads;   // packs of a thread
  static_assert(kBatch % 2 == 0, "a batch is whole loads");
#pragma unroll 1
  for (int b = 0; b < row.batches; ++b) {
    unsigned long long s = 0;
#pragma unroll 1
    for (int i = b * kBatch; i < min(most, (b + 1) * kBatch); i += 4) {
      uint4 raw[4];
      row.load(raw, i);
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
        s += of_pack(raw[0], row.elem(0, i + 2 * h)) + of_pack(raw[1], row.elem(0, i + 2 * h + 1));
        raw[0] = raw[2];
        raw[1] = raw[3];
      }
    }
    if (!__any_sync(0xffffffffu, s != 0)) continue;
    s = warp_reduce(s, AddOp());
    if (row.lane == 0) atomicAdd(&sh.rec[b], s);
  }
  __syncthreads();
  unsigned long long total = 0;
  for (int b = 0; b < row.batches; ++b) total += sh.rec[b];
  const int count = counted(f);   // of the first sweep; what the search adds is not wanted
  const unsigned long long n = nth(total);
  unsigned long long before = 0;
  int b = 0;
  while (b < row.batches - 1 && before + sh.rec[b] < n) before += sh.rec[b++];
#pragma unroll 1
  for (int j = 0; j < kBatch; ++j) {
    const unsigned long long s =
        warp_reduce(of_pack(row.load_one(b * kBatch + j), row.elem(b, j)), AddOp());
    if (row.lane == 0) sh.grid[j * kWarps + row.warp] = s;
  }
  __syncthreads();
  int at = 0;
  while (at < kBatch * kWarps - 1 && before + sh.grid[at] < n) before += sh.grid[at++];
  if (row.warp == at % kWarps) {
    const int j = at / kWarps;
    const uint4 p = row.load_one(b * kBatch + j);
    const unsigned long long mine = of_pack(p, row.elem(b, j));
    unsigned long long incl = warp_scan(mine);
    unsigned long long run = before + incl - mine;
    if (run < n && n <= run + mine)
      for (int e = 0; e < kPerPack<E>; ++e) {
        const int id = row.elem(b, j) + e;
        const unsigned long long t = f(pack_elem_at<E>(p, e), id);
        if (run < n && n <= run + t) {
          sh.found = uint32_t(id);
          sh.kept = t;
        }
        run += t;
      }
  }
  __syncthreads();
  const Found r{int(uint32_t(sh.found)), sh.kept, total, count};
  __syncthreads();   // before `found` and `rec` are written again
  return r;
}

// Radix select among the tokens that `cut` keeps: the largest key at which the summed weights, from
// the largest key down, no longer satisfy need(sum); need(0) may be false (then the first key).
// weight: up to 2^31.  need.set() gets the sum of all weights before the first choice.
struct Selected {
  uint32_t key;
  unsigned long long above, total;   // sums over larger keys, over all
};
template <typename R, typename W, typename Need>
ALR_DEV Selected select_key(R& row, const Cut& cut, W weight, Need need) {
  using E = typename R::E;
  Shared& sh = row.sh;
  // a bf16 key is in the upper 16 bits, the low ones follow from the sign
  constexpr int kLevels = sizeof(E) == 2 ? 2 : 3;
  constexpr int kShift[3] = {21, sizeof(E) == 2 ? 16 : 10, 0};
  uint32_t prefix = 0;
  unsigned long long above = 0, total = 0;
  const int tid = threadIdx.x, threads = blockDim.x;
  for (int level = 0; level < kLevels; ++level) {
    const int shift = kShift[level], up = level == 0 ? 32 : kShift[level - 1];
    const uint32_t mask = (1u << (up - shift)) - 1u;
    const int bins = int(mask) + 1;
    for (int b = tid; b < bins; b += threads) sh.many.lo[b] = sh.many.hi[b] = 0;
    __syncthreads();
    row.each_heavy([&](const uint4& p, int id) {
#pragma unroll 1
      for (int e = 0; e < kPerPack<E>; ++e) {
        const float x = pack_elem_at<E>(p, e);
        if (!(x > kNegInf)) continue;
        const uint32_t k = order_key(x);
        if (level > 0 && (k ^ prefix) >> up != 0) continue;
        if (!cut.keeps(k, id + e)) continue;
        const uint32_t w = weight(x);
        if (w != 0) add_bin(sh, (k >> shift) & mask, w);
      }
    });
    row.sync();
    total_bins(row, bins);
    // from the largest bin down: thread t takes the bins [bins - 1 - t n, ...) downwards
    const int n = (bins + threads - 1) / threads;
    unsigned long long mine = 0;
    for (int j = 0; j < n; ++j) {
      const int b = bins - 1 - (tid * n + j);
      if (b >= 0) mine += sh.many.total[b];
    }
    unsigned long long incl = warp_scan(mine);
    if (row.lane == 31) sh.lbuf[row.warp] = incl;
    __syncthreads();
    unsigned long long run = above + incl - mine, all = 0;
    for (int w = 0; w < row.n_warps; ++w) {
      if (w < row.warp) run += sh.lbuf[w];
      all += sh.lbuf[w];
    }
    if (level == 0) {
      total = all;
      need.set(all);
    }
    for (int j = 0; j < n; ++j) {
      const int b = bins - 1 - (tid * n + j);
      if (b < 0) break;
      const unsigned long long t = sh.many.total[b];
      if (t != 0 && (run == above ? (above == 0 || need(run)) : need(run)) && !need(run + t)) {
        sh.digit = uint32_t(b);
        sh.above = run;
      }
      run += t;
    }
    __syncthreads();
    prefix |= sh.digit << shift;
    above = sh.above;
    __syncthreads();
  }
  if (sizeof(E) == 2 && !(prefix >> 31)) prefix |= 0xffffu;   // negative: the low bits are inverted
  return {prefix, above, total};
}

// The last id kept of the tokens with `key` that `cut` keeps, n (>= 1) of them.
template <typename R>
ALR_DEV int nth_equal(R& row, const Cut& cut, uint32_t key, unsigned long long n) {
  const auto is = [&](float x, int v) -> unsigned long long {
    return x > kNegInf && order_key(x) == key && cut.keeps(key, v);
  };
  const Found f = find_unit(
      row, key_value(key), OfPack<typename R::E, decltype(is)>{is},
      [n](unsigned long long total) { return n < total ? n : total; });
  return f.id;
}

// What a cut is asked for: k tokens, or the share p of a mass.  reach(): how many tokens of weight w each,
// one at least, after a sum `above`.
struct NeedCount {
  unsigned long long k;
  ALR_DEV void set(unsigned long long) {}
  ALR_DEV unsigned long long reach(unsigned long long above, unsigned long long) const {
    return k - above;
  }
  ALR_DEV bool operator()(unsigned long long got) const { return got < k; }
};
struct NeedMass {
  double p, lim;
  ALR_DEV void set(unsigned long long total) { lim = p * double(total); }
  ALR_DEV unsigned long long reach(unsigned long long above, unsigned long long w) const {
    const double want = (lim - double(above)) / double(w);
    unsigned long long n = want < 1.0 ? 1ull : (unsigned long long)want;
    while (n > 1 && !(double(above + (n - 1) * w) < lim)) --n;
    while (double(above + n * w) < lim) ++n;
    return n;
  }
  ALR_DEV bool operator()(unsigned long long got) const { return double(got) < lim; }
};

// The cut that keeps the k first candidates of the row, which has more.
template <typename R>
ALR_DEV Cut cut_top_k(R& row, int k) {
  const Cut all{0u, 0x7fffffff};
  NeedCount need{(unsigned long long)k};
  const Selected s = select_key(row, all, [](float) { return 1u; }, need);
  return {s.key, nth_equal(row, all, s.key, k - s.above)};
}

// A lower bound of the row's K-th largest logit that few more reach (-inf when the threads hold too few),
// and the largest logit.  All blocks get both.
struct Bound {
  float least, top;
};
template <typename R>
ALR_DEV Bound row_bound(R& row, int K) {
  using E = typename R::E;
  Shared& sh = row.sh;
  float t = kNegInf;
  row.each_first([&](const uint4& p, int) { t = fmaxf(t, largest<E>(p)); });
  row.most = t;
  // the `per` largest of the warp's 32, into all blocks' lists
  const int n_rec = row.records(), tid = threadIdx.x, threads = blockDim.x;
  const int per = K > 1 ? min(32, (K + n_rec - 1) / n_rec + 1) : 1, n = n_rec * per;
  row.ready();
  if (tid == 0) sh.n_more = 0;
  if (n > kListWarp)
    for (int i = tid; i < 256; i += threads) sh.small[i] = 0;
  for (int j = 0; j < per; ++j) {
    const float m = warp_max(t);
    row.to_all(&sh.few.list[row.record() * per + j], m);
    const unsigned who = __ballot_sync(0xffffffffu, t == m);
    if (row.lane == __ffs(who) - 1) t = kNegInf;
  }
  row.sync();
  float top = kNegInf;
  for (int i = row.lane; i < n_rec; i += 32) top = fmaxf(top, sh.few.list[i * per]);
  top = warp_max(top);
  if (K <= 1) {
    __syncthreads();   // every warp has read the list: a histogram is cleared over it next
    return {K == 1 ? top : kNegInf, top};
  }
  if (n <= kListWarp) {   // the upper half of the K-th largest key, bit by bit
    if (row.warp == 0) {
      uint32_t key[kListWarp / 32], least = 0;
#pragma unroll
      for (int j = 0; j < kListWarp / 32; ++j) {
        const int i = j * 32 + row.lane;
        const float v = i < n ? sh.few.list[i] : kNegInf;
        key[j] = v > kNegInf ? order_key(v) >> 16 : 0u;
      }
#pragma unroll 1
      for (uint32_t bit = 0x8000u; bit != 0; bit >>= 1) {
        int reach = 0;
#pragma unroll
        for (int j = 0; j < kListWarp / 32; ++j)
          if (j * 32 < n) reach += __popc(__ballot_sync(0xffffffffu, key[j] >= (least | bit)));
        if (reach >= K) least |= bit;
      }
      if (row.lane == 0) sh.digit = least;
    }
    __syncthreads();
    return {sh.digit != 0 ? key_value(sh.digit << 16) : kNegInf, top};
  }
  // the upper half of the K-th largest key, 8 bits at a time
  uint32_t prefix = 0, reach = uint32_t(K);
  for (int shift = 24; shift >= 16; shift -= 8) {
    for (int i = tid; i < n; i += threads) {
      const float v = sh.few.list[i];
      const uint32_t key = order_key(v);
      if (v > kNegInf && (shift == 24 || key >> 24 == prefix >> 24))
        atomicAdd(&sh.small[(key >> shift) & 255], 1u);
    }
    __syncthreads();
    if (row.warp == 0) {   // lane l: the bins 255 - 8 l and the seven below
      uint32_t mine = 0;
      for (int j = 0; j < 8; ++j) mine += sh.small[255 - 8 * row.lane - j];
      uint32_t incl = warp_scan(mine);
      if (row.lane == 31) sh.digit = incl >= reach ? 0u : 0xffffffffu;   // too few
      __syncwarp();
      uint32_t run = incl - mine;
      if (run < reach && incl >= reach) {
        int b = 255 - 8 * row.lane;
        while (run + sh.small[b] < reach) run += sh.small[b--];
        sh.digit = uint32_t(b);
        sh.reach = reach - run;
      }
    }
    __syncthreads();
    if (sh.digit == 0xffffffffu) return {kNegInf, top};
    prefix |= sh.digit << shift;
    reach = sh.reach;
    for (int i = tid; i < 256; i += threads) sh.small[i] = 0;
    __syncthreads();
  }
  return {key_value(prefix), top};
}

// Sends the entries that take(x, id) wants, of those in [least, most], to the cluster's first block: a
// warp's first ones into its own places there, more of them to places that it asks for.  All blocks are
// in step afterwards.
template <bool kHeavy = false, typename R, typename F>
ALR_DEV void collect(R& row, float least, float most, F take) {
  using E = typename R::E;
  Shared& sh = row.sh;
  int total = 0;
  const bool has = row.most >= least && row.most > kNegInf;
  if (__any_sync(0xffffffffu, has)) {
    const auto each = [&](auto f) {
      if (!has) return;
      const auto of_pack = [&](const uint4& p, int id) {
        const float m = largest<E>(p);
        if (!(m >= least) || !(m > kNegInf)) return;
        uint32_t bits = 0;
#pragma unroll
        for (int e = 0; e < kPerPack<E>; ++e) {
          const float x = pack_elem<E>(p, e);
          bits |= uint32_t(x >= least && x <= most && x > kNegInf) << e;
        }
        for (; bits != 0; bits &= bits - 1) {
          const int e = __ffs(bits) - 1;
          const float x = pack_elem_at<E>(p, e);
          if (take(x, id + e)) f(entry(order_key(x), id + e));
        }
      };
      if constexpr (kHeavy)
        row.each_heavy(of_pack);
      else
        row.each(of_pack);
    };
    int mine = 0;
    unsigned long long first = 0, second = 0;
    each([&](unsigned long long e) {
      if (mine == 0) first = e;
      if (mine == 1) second = e;
      ++mine;
    });
    int at = warp_scan(mine);
    total = __shfl_sync(0xffffffffu, at, 31);
    at -= mine;
    int more = 0;
    if (total > kSlots) {
      if (row.lane == 0) more = row.add_first(&sh.n_more, total - kSlots);
      more = __shfl_sync(0xffffffffu, more, 0) + row.records() * kSlots - kSlots;
    }
    const auto send = [&](unsigned long long e) {
      const int to = at < kSlots ? row.record() * kSlots + at : more + at;
      if (to < kCandMost) row.to_first(&sh.cand[to], e);
      ++at;
    };
    if (__any_sync(0xffffffffu, mine > 2)) {
      each(send);
    } else {
      if (mine > 0) send(first);
      if (mine > 1) send(second);
    }
  }
  if (row.lane == 0) row.to_first(&sh.count[row.record()], min(total, kSlots));
  row.sync();
}

// row_bound and collect in one reading of the row by one block: the K-th largest of the threads' largest
// logits, once the first packs are there (and again after the next ones), is a bound that every later pack is
// held against as it comes by.  768 x 151936 rows, us, in one reading and as row_bound and collect: top 64
// 167 and 182, top 256 236 and 296, tokens of a top-k of 64 85 and 155, of 256 146 and 197.
template <typename R>
ALR_DEV Bound bound_and_collect(R& row, int K) {
  if constexpr (std::is_base_of_v<RowCommon<true>, R>) {
    using E = typename R::E;
    static_assert(kTopMost <= kStreamThreads, "a thread's largest for each of the K");
    Shared& sh = row.sh;
    constexpr int kBatch = R::kBatch;
    row.ready();
    if (threadIdx.x == 0) sh.n_more = 0;
    for (int i = threadIdx.x; i < row.records(); i += blockDim.x) sh.count[i] = 0;
    __syncthreads();
    float most = kNegInf, least = kNegInf;
    for (int b = 0; b < row.batches; ++b) {
      uint4 raw[kBatch];
      row.load(raw, b * kBatch);
      float top[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        top[j] = largest<E>(raw[j]);
        most = fmaxf(most, top[j]);
      }
      // Bit by bit of the upper half of the keys.  For few tokens the bound rises little after two batches (top
      // 8: 109 us, 114 with a bound in every batch; top 64 167 and 150, a token of its top-k 85 and 92), for many it
      // does (top 96: 170, 193 without).  Rows that rise from end to end overflow it and take the radix select:
      // 903 us for the top 64 of 768, 699 for tokens of a top-k.
      if (b < 2 || K > 64 || least == kNegInf) {
        const uint32_t key = most > kNegInf ? order_key(most) >> 16 : 0u;
        uint32_t bound = 0;
        for (uint32_t bit = 0x8000u; bit != 0; bit >>= 1)
          if (__syncthreads_count(key >= (bound | bit)) >= K) bound |= bit;
        if (bound != 0) least = key_value(bound << 16);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (!(top[j] >= least) || !(top[j] > kNegInf)) continue;
        uint32_t bits = 0;
#pragma unroll
        for (int e = 0; e < kPerPack<E>; ++e)
          bits |= uint32_t(pack_elem<E>(raw[j], e) >= least && pack_elem<E>(raw[j], e) > kNegInf) << e;
        int at = row.records() * kSlots + atomicAdd(&sh.n_more, __popc(bits));
        for (; bits != 0; bits &= bits - 1, ++at) {
          const int e = __ffs(bits) - 1;
          if (at < kCandMost)
            sh.cand[at] = entry(order_key(pack_elem_at<E>(raw[j], e)), row.elem(b, j) + e);
        }
      }
    }
    row.most = most;
    const float top = block_reduce(most, MaxOp(), sh.fbuf);   // and all candidates are there
    return {least, top};
  } else {
    const Bound b = row_bound(row, K);
    if (b.top > kNegInf) collect(row, b.least, -kNegInf, [](float, int) { return true; });
    return b;
  }
}

// Whether all candidates fit, known to all blocks.  The others then wait in the cluster barrier until all
// have read it; the first block arrives at once and waits (others_know) when it likes to.
ALR_DEV bool candidates_fit(const RowCommon<true>& row) {
  const bool fit = row.records() * kSlots + row.sh.n_more <= kCandMost;
  if (!fit) __syncthreads();   // all have read it: what the block does then begins with setting it to 0
  return fit;
}
ALR_DEV void others_know(const RowCommon<true>&) {}
ALR_DEV bool candidates_fit(const RowCommon<false>& row) {
  const int n = row.rank == 0 ? row.sh.n_more : ld_cluster_s32(cluster_smem_addr(&row.sh.n_more, 0));
  const bool fit = row.records() * kSlots + n <= kCandMost;
  cluster_arrive();
  if (row.rank != 0 || !fit) cluster_wait();
  return fit;
}
ALR_DEV void others_know(const RowCommon<false>& row) {
  if (row.rank == 0) cluster_wait();
}

// First block: the candidates in order, in few.all; returns their number.
template <typename R>
ALR_DEV int sort_candidates(R& row) {
  Shared& sh = row.sh;
  const int tid = threadIdx.x, threads = blockDim.x, n_rec = row.records();
  if (row.warp == 0) {   // offsets of the warps' places: lane l has the records [4 l, 4 l + 4)
    static_assert(kWarpsMost <= 128, "four records a lane");
    int c[4], mine = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      c[j] = row.lane * 4 + j < n_rec ? sh.count[row.lane * 4 + j] : 0;
      mine += c[j];
    }
    int at = warp_scan(mine);
    if (row.lane == 31) sh.kept_n = at;
    at -= mine;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (row.lane * 4 + j < n_rec) sh.count[row.lane * 4 + j] = at;
      at += c[j];
    }
    if (row.lane == 31) sh.count[n_rec] = sh.kept_n;
  }
  __syncthreads();
  const int base = sh.count[n_rec], n = base + sh.n_more;
  unsigned long long *to = sh.few.all, *raw = n <= kCandSort ? to + kCandSort : to;
  for (int i = tid; i < n_rec * kSlots; i += threads) {
    const int w = i / kSlots, j = i % kSlots;
    if (sh.count[w] + j < sh.count[w + 1]) raw[sh.count[w] + j] = sh.cand[i];
  }
  for (int i = tid; i < sh.n_more; i += threads) raw[base + i] = sh.cand[n_rec * kSlots + i];
  if (n <= kCandSort) {
    __syncthreads();
    // eight lanes count for an entry
    for (int i0 = 0; i0 < n; i0 += threads / 8) {
      const int i = i0 + tid / 8;
      const unsigned long long v = i < n ? raw[i] : 0ull;
      int place = 0;
      for (int j = tid & 7; j < n; j += 8) place += raw[j] > v;
#pragma unroll
      for (int off = 4; off > 0; off >>= 1) place += __shfl_xor_sync(0xffffffffu, place, off);
      if ((tid & 7) == 0 && i < n) to[place] = v;
    }
    __syncthreads();
    return n;
  }
  int size = 2 * kCandSort;
  while (size < n) size *= 2;
  for (int i = n + tid; i < size; i += threads) to[i] = 0ull;
  __syncthreads();
  for (int k = 2; k <= size; k *= 2)
    for (int j = k / 2; j > 0; j /= 2) {
      for (int p = tid; p < size / 2; p += threads) {
        const int a = 2 * p - (p & (j - 1)), b = a + j;
        const unsigned long long u = to[a], v = to[b];
        if ((u < v) == ((a & k) == 0)) {
          to[a] = v;
          to[b] = u;
        }
      }
      __syncthreads();
    }
  return n;
}

// ---------------------------------------------------------------- top logits ---
struct TopOut {
  float* val;
  int32_t* idx;
  float* lse;
  float* lse_rest;
};

template <typename R>
__device__ __noinline__ Cut exact_top_k(R row, int K) {
  return cut_top_k(row, K);
}

template <typename R>
ALR_DEV void top_logits_row(R& row, int K, float t, const TopOut& out, long long r) {
  using E = typename R::E;
  Shared& sh = row.sh;
  const Bound bound = bound_and_collect(row, K);
  Cut cut{0u, -1};
  if (!(bound.top > kNegInf)) {   // nothing to list; all blocks agree, none reads another's memory
    for (int i = threadIdx.x; row.rank == 0 && i < K; i += blockDim.x) {
      out.val[r * K + i] = kNegInf;
      out.idx[r * K + i] = -1;
    }
    if (row.rank == 0 && threadIdx.x == 0) {
      if (out.lse != nullptr) out.lse[r] = kNegInf;
      if (out.lse_rest != nullptr) out.lse_rest[r] = kNegInf;
    }
    return;
  }
  if (!candidates_fit(row)) {   // more than fit reach the bound: find the exact cut
    cut = exact_top_k(row, K);
    if (threadIdx.x == 0) sh.n_more = 0;
    row.sync();
    collect(row, key_value(cut.key), -kNegInf, [&](float x, int v) { return cut.keeps(order_key(x), v); });
    (void)candidates_fit(row);
  }
  others_know(row);   // the records below go over the cluster
  // The others' sums, each warp's from its own largest; the candidates are the first block's.
  const float k = 1.f / t * kLog2e, least = cut.last >= 0 ? key_value(cut.key) : bound.least;
  const auto without = [&](uint4 p, int id) {
    if (largest<E>(p) >= least) {
      uint32_t bits = 0;
#pragma unroll 1
      for (int e = 0; e < kPerPack<E>; ++e) {
        const float x = pack_elem_at<E>(p, e);
        const bool taken =
            x >= least && (cut.last < 0 || cut.keeps(x > kNegInf ? order_key(x) : 0u, id + e));
        bits |= uint32_t(taken) << e;
      }
      mask_pack<E>(p, bits);
    }
    return p;
  };
  float m = kNegInf;
  if constexpr (std::is_base_of_v<RowCommon<true>, R>) {
    m = least;   // read once more, not twice: from the bound, or again if that is too far above
  } else {
    row.each([&](uint4& p, int id) {
      p = without(p, id);
      m = fmaxf(m, largest<E>(p));
    });
    m = warp_max(m);
  }
  const auto sum_from = [&](float ref) {
    const uint64_t m2 = f2_pack(ref, ref), k2 = f2_pack(k, k);
    uint64_t s2 = 0;
    row.each([&](const uint4& q, int id) {
      uint4 p = q;
      if constexpr (std::is_base_of_v<RowCommon<true>, R>) p = without(q, id);
#pragma unroll
      for (int e = 0; e < kPerPack<E>; e += 2)
        s2 = f2_add(s2, f2_ex2(f2_mul(f2_sub(f2_pack(pack_elem<E>(p, e), pack_elem<E>(p, e + 1)), m2),
                                      k2)));
    });
    float a, b;
    f2_unpack(s2, a, b);
    return warp_reduce(a + b, AddOp());
  };
  float s = m > kNegInf ? sum_from(m) : 0.f;
  if constexpr (std::is_base_of_v<RowCommon<true>, R>) {
    // An exponent of -n octaves is rounded to n 2^-24: from a reference far above the rest its sum would lose
    // what the cluster form, which takes each warp's own largest, does not.  20 octaves: the rest of a trained row
    // under its first token mostly reaches that (top 1 of 768 x 151936: 112 us; 187 with a limit of 8 octaves, which
    // has most warps read twice more).  (The same in the whole warp.)
    if (m > kNegInf && !(s > 0x1p-20f)) {
      m = kNegInf;
      row.each([&](const uint4& p, int id) { m = fmaxf(m, largest<E>(without(p, id))); });
      m = warp_max(m);
      s = m > kNegInf ? sum_from(m) : 0.f;
    }
    if (!(s > 0.f)) m = kNegInf;
  }
  row.to_all(&sh.frec[row.record()], make_float2(m, s));
  row.sync();   // no other block's memory is read any more
  if (row.rank == 0) {
    const int n = sort_candidates(row);
    const int tid = threadIdx.x, threads = blockDim.x, got = min(n, K);
    for (int i = tid; i < K; i += threads) {
      out.val[r * K + i] = i < got ? key_value(entry_key(sh.few.all[i])) : kNegInf;
      out.idx[r * K + i] = i < got ? entry_id(sh.few.all[i]) : -1;
    }
    // the rest: candidates past the K first, and all others (who have the candidates below `least`, which
    // a streamed row collected before its bound rose)
    float mo = kNegInf;
    for (int i = K + tid; i < n; i += threads) {
      const float v = key_value(entry_key(sh.few.all[i]));
      if (v >= least) mo = fmaxf(mo, v);
    }
    for (int i = tid; i < row.records(); i += threads) mo = fmaxf(mo, sh.frec[i].x);
    mo = block_reduce(mo, MaxOp(), sh.fbuf);
    float so = 0.f, sl = 0.f;
    if (mo > kNegInf) {
      for (int i = K + tid; i < n; i += threads) {
        const float v = key_value(entry_key(sh.few.all[i]));
        if (v >= least) so += ex2((v - mo) * k);
      }
      for (int i = tid; i < row.records(); i += threads)
        if (sh.frec[i].x > kNegInf) so += sh.frec[i].y * ex2((sh.frec[i].x - mo) * k);
    }
    so = block_reduce(so, AddOp(), sh.fbuf);
    for (int i = tid; i < got; i += threads)
      sl += ex2((key_value(entry_key(sh.few.all[i])) - bound.top) * k);
    sl = block_reduce(sl, AddOp(), sh.fbuf);
    if (tid == 0) {
      const bool any = mo > kNegInf;
      if (any) sl += so * ex2((mo - bound.top) * k);
      if (out.lse != nullptr) out.lse[r] = n > 0 ? bound.top / t + logf(sl) : kNegInf;
      if (out.lse_rest != nullptr) out.lse_rest[r] = any ? mo / t + logf(so) : kNegInf;
    }
  }
}

template <typename E, int kPacks>
__global__ void __launch_bounds__(kRowThreadsMost, kPacks > 10 ? 1 : 2)
    top_logits_kernel(const E* Z, long long ldz, int V, int K, float t, TopOut out, int cluster) {
  __shared__ Shared sh;
  pdl_wait_and_release();
  const long long r = cluster_id_x();
  Row<E, kPacks> row(Z + r * ldz, r * ldz, V, cluster, sh);
  top_logits_row(row, K, t, out, r);
}

template <typename E>
__global__ void __launch_bounds__(kStreamThreads, 2)
    top_logits_stream_kernel(const E* Z, long long N, long long ldz, int V, int K, float t,
                             TopOut out) {
  __shared__ Shared sh;
  pdl_wait_and_release();
  for (long long r = blockIdx.x; r < N; r += gridDim.x) {
    StreamRow<E> row(Z + r * ldz, r * ldz, V, sh);
    top_logits_row(row, K, t, out, r);
  }
}

// ------------------------------------------------------------------ sampling ---
// A token's weight is the whole number floor(2^31 exp2((z - max) c)), c = log2 e / temperature, every
// step rounded to fp32 on its own: sums of weights are exact, so neither the order of summation nor
// the split of a row over threads can change a draw.
struct Weight {
  float m, c;
  // exp2f and ex2.approx agree where the weight is not 0 (all 1.1e9 floats of [-64, 0] were compared)
  ALR_DEV float real(float x) const { return ex2(__fmul_rn(__fsub_rn(x, m), c)); }
  // Logits below have a real weight under w (and above: not certainly over it); with a margin for the
  // rounding of the three steps.
  ALR_DEV float below(float w) const {
    const float d = (log2f(w) - 0.01f) / c;
    return d == d ? m + d - 1e-6f * fabsf(m) : kNegInf;
  }
  ALR_DEV uint32_t operator()(float x) const { return __float2uint_rz(real(x) * 2147483648.f); }
};

struct SampleOut {
  int32_t* token;
  float* prob;
  int32_t* n_kept;
  ALR_DEV void put(long long r, int t, float p, int n) const {
    token[r] = t;
    if (prob != nullptr) prob[r] = p;
    if (n_kept != nullptr) n_kept[r] = n;
  }
};

// First block: draws from the n <= kTopMost first tokens of the row, in order in few.all.
ALR_DEV void draw_from_candidates(Shared& sh, int n, const Weight& weight, float top_p, float min_p,
                                  uint32_t u, long long r, const SampleOut& out) {
  const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 31;
  unsigned long long* w = sh.few.w;
  for (int i = tid; i < n; i += threads) w[i] = weight(key_value(entry_key(sh.few.all[i])));
  __syncthreads();
  if (tid < 32) {   // lane l: the tokens [8 l, 8 l + 8); kept is a prefix
    constexpr int kOwn = kTopMost / 32;
    unsigned long long own[kOwn], mine = 0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      own[j] = lane * kOwn + j < n ? w[lane * kOwn + j] : 0ull;
      mine += own[j];
    }
    unsigned long long incl = warp_scan(mine);
    const unsigned long long sum = __shfl_sync(0xffffffffu, incl, 31);
    // the sum before a token, a whole number, is below top_p sum: below that number rounded up
    const unsigned long long lim =
        top_p >= 1.f ? ~0ull : (unsigned long long)ceil(fmax(double(top_p), 0.0) * double(sum));
    unsigned long long before = incl - mine, S = 0;
    int kept = 0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const int i = lane * kOwn + j;
      const bool keep = own[j] != 0 && (i == 0 || (before < lim &&
                        weight.real(key_value(entry_key(sh.few.all[min(i, n - 1)]))) >= min_p));
      before += own[j];
      if (keep) {
        S += own[j];
        ++kept;
      }
    }
    S = warp_reduce(S, AddOp());
    kept = __reduce_add_sync(0xffffffffu, kept);
    if (lane == 0) {
      sh.kept = S;
      sh.kept_n = kept;
    }
  }
  __syncthreads();
  const int kept = sh.kept_n;
  const unsigned long long S = sh.kept, target = __umul64hi((unsigned long long)u << 32, S);
  // the kept weight before each token in the order of ids: eight lanes add it up
  for (int i0 = 0; i0 < kept; i0 += threads / 8) {
    const int i = i0 + tid / 8;
    const uint32_t id = i < kept ? uint32_t(entry_id(sh.few.all[i])) : 0u;
    unsigned long long before = 0;
    for (int j = tid & 7; j < kept; j += 8)
      before += uint32_t(entry_id(sh.few.all[j])) < id ? w[j] : 0ull;
#pragma unroll
    for (int off = 4; off > 0; off >>= 1) before += __shfl_xor_sync(0xffffffffu, before, off);
    if ((tid & 7) == 0 && i < kept && before <= target && target < before + w[i])
      out.put(r, int(id), float(double(w[i]) / double(S)), kept);
  }
}

// Even steps of the logit below the largest, kBins over the 32 octaves below which weights are 0.  The
// conversion takes anything below 0 to 0: no logit has a place outside the bins.
struct Steps {
  float top, scale;
  ALR_DEV int operator()(float x) const {
    return int(min(uint32_t(kBins - 1), __float2uint_rz((top - x) * scale)));
  }
};

// The cut that keeps, of the tokens of positive weight that `cut` keeps, the first ones whose summed worth
// need() still asks for before them (one at least); `cut` itself when need() is content with all of them.
// worth: 0 .. 2^31 for x, 0 where the weight is 0, as it is below `least`.
// The histogram is of the logits that reach `near` first: a trained model's nucleus ends among those few,
// and a place in a histogram is what costs most here.  Where it goes on, all logits have one.  A nucleus of 768 x
// 151936 trained rows, us, with 16 octaves first and all 32 at once: 245 and 240 at a temperature of 0.8, 265 and
// 438 at 1, 266 and 560 at 1.3, 752 and 627 at 1.6, where it takes in the bulk; of a random head 740 and 696.
template <typename R, typename W, typename Need>
ALR_DEV Cut cut_by_steps(R& row, const Cut& cut, const Steps& bin, float least, float near, W worth,
                         Need need) {
  using E = typename R::E;
  Shared& sh = row.sh;
  const int tid = threadIdx.x, threads = blockDim.x;
  const float lowest = fmaxf(least, key_value(cut.key));
  const bool cut_any = cut.key != 0;
  const int n = (kBins + threads - 1) / threads;
  unsigned long long run = 0;
  for (float from = fmaxf(near, lowest);; from = lowest) {
    for (int b = tid; b < kBins; b += threads) sh.many.lo[b] = sh.many.hi[b] = 0;
    if (tid == 0) {
      sh.n_more = 0;
      sh.digit = 0xffffffffu;
    }
    __syncthreads();
    unsigned long long below = 0;   // what has no place in the histogram
    row.each_heavy([&](const uint4& p, int id) {
      const bool some = largest<E>(p) >= lowest;
      const int lanes = __popc(__ballot_sync(0xffffffffu, some));
      const auto place = [&](float x, int v, uint32_t w) {
        if (w != 0 && (!cut_any || cut.keeps(order_key(x), v))) add_bin(sh, bin(x), w);
      };
      if (from > lowest && lanes >= 8) {
        uint32_t bits = 0;
#pragma unroll
        for (int e = 0; e < kPerPack<E>; ++e) {
          const float x = pack_elem<E>(p, e);
          const uint32_t w = worth(x);
          below += x >= from ? 0u : w;
          bits |= uint32_t(x >= from) << e;
        }
        for (; bits != 0; bits &= bits - 1) {
          const int e = __ffs(bits) - 1;
          const float x = pack_elem_at<E>(p, e);
          place(x, id + e, worth(x));
        }
      } else if (some) {
        for (uint32_t bits = reaching<E>(p, lowest); bits != 0; bits &= bits - 1) {
          const int e = __ffs(bits) - 1;
          const float x = pack_elem_at<E>(p, e);
          const uint32_t w = worth(x);
          if (x >= from)
            place(x, id + e, w);
          else
            below += w;
        }
      }
    });
    below = warp_reduce(below, AddOp());
    row.to_all(&sh.rec[row.record()], below);
    row.sync();
    total_bins(row, kBins);
    unsigned long long mine = 0;
    for (int j = tid * n; j < min(kBins, (tid + 1) * n); ++j) mine += sh.many.total[j];
    unsigned long long incl = warp_scan(mine);
    if (row.lane == 31) sh.lbuf[row.warp] = incl;
    __syncthreads();
    run = incl - mine;
    unsigned long long placed = 0, rest = 0;
    for (int w = 0; w < row.n_warps; ++w) {
      if (w < row.warp) run += sh.lbuf[w];
      placed += sh.lbuf[w];
    }
    for (int i = row.lane; i < row.records(); i += 32) rest += sh.rec[i];
    rest = warp_reduce(rest, AddOp());
    need.set(placed + rest);
    // (what follows is the same in all threads of the cluster)
    if (!need(placed)) break;
    if (from == lowest) return cut;   // all of them
    row.sync();
  }
  for (int j = tid * n; j < min(kBins, (tid + 1) * n); ++j) {
    const unsigned long long t = sh.many.total[j];
    if (t != 0 && (run == 0 || need(run)) && !need(run + t)) {
      sh.digit = uint32_t(j);
      sh.above = run;
    }
    run += t;
  }
  __syncthreads();
  const int step = int(sh.digit);
  const unsigned long long above = sh.above;
  // that step's tokens, in order
  const float hi = bin.top - float(step) / bin.scale, lo = bin.top - float(step + 1) / bin.scale;
  const float wide = 1e-6f * (fabsf(bin.top) + fabsf(lo)) + 0.01f / bin.scale;   // for the roundings
  collect<true>(row, lo - wide > lowest && step < kBins - 1 ? lo - wide : lowest,
                hi + wide < -kNegInf ? hi + wide : -kNegInf, [&](float x, int v) {
    return bin(x) == step && worth(x) != 0 && (!cut_any || cut.keeps(order_key(x), v));
  });
  if (!candidates_fit(row)) {   // too many of them
    const Selected s = select_key(row, cut, worth, need);
    return {s.key, nth_equal(row, cut, s.key, need.reach(s.above, worth(key_value(s.key))))};
  }
  others_know(row);
  if (row.rank == 0) {
    const int got = sort_candidates(row);
    // the last token before which need() asks for more
    const int m = (got + threads - 1) / threads;
    unsigned long long own = 0;
    for (int i = tid * m; i < min(got, (tid + 1) * m); ++i)
      own += worth(key_value(entry_key(sh.few.all[i])));
    unsigned long long in = warp_scan(own);
    if (row.lane == 31) sh.lbuf[row.warp] = in;
    __syncthreads();
    unsigned long long at = above + in - own;
    for (int w = 0; w < row.warp; ++w) at += sh.lbuf[w];
    for (int i = tid * m; i < min(got, (tid + 1) * m); ++i) {
      const unsigned long long w = worth(key_value(entry_key(sh.few.all[i])));
      if ((at == 0 || need(at)) && !need(at + w)) sh.found = sh.few.all[i];
      at += w;
    }
    __syncthreads();
    if (row.warp == 0) row.to_all(&sh.kept, sh.found);
  }
  row.sync();
  const unsigned long long last = sh.kept;
  row.sync();
  return {entry_key(last), entry_id(last)};
}

// Weights of the tokens kept: those above `edge`, at it up to id `last`, of a real weight of min_p at least.
template <typename E>
struct Mass {
  Weight weight;
  float edge;
  int last;
  float min_p;
  int count;   // of tokens in the packs summed up
  ALR_DEV unsigned long long operator()(float x, int id) const {
    if (!(x > edge || (x == edge && id <= last))) return 0;
    const float w = weight.real(x);
    return w >= min_p || x == weight.m ? __float2uint_rz(w * 2147483648.f) : 0u;
  }
  ALR_DEV unsigned long long few(const uint4& p, int id, float least) {
    unsigned long long s = 0;
    for (uint32_t bits = reaching<E>(p, least); bits != 0; bits &= bits - 1) {
      const int e = __ffs(bits) - 1;
      const unsigned long long q = (*this)(pack_elem_at<E>(p, e), id + e);
      s += q;
      count += q != 0;
    }
    return s;
  }
  ALR_DEV unsigned long long pack(const uint4& p, int id, float) {
    unsigned long long s = 0;
    bool at_edge = false;
#pragma unroll
    for (int e = 0; e < kPerPack<E>; ++e) {
      const float x = pack_elem<E>(p, e), w = weight.real(x);
      uint32_t q = __float2uint_rz(w * 2147483648.f);
      if (!(x >= edge) || !(w >= min_p || x == weight.m)) q = 0;
      at_edge |= x == edge;
      s += q;
      count += q != 0;
    }
    if (at_edge && id + kPerPack<E> > last)   // tokens at the edge, some past the last one
#pragma unroll 1
      for (int e = 0; e < kPerPack<E>; ++e) {
        const float x = pack_elem_at<E>(p, e);
        if (!(x == edge) || id + e <= last) continue;
        const float w = weight.real(x);
        const uint32_t q = w >= min_p || x == weight.m ? __float2uint_rz(w * 2147483648.f) : 0u;
        s -= q;
        count -= q != 0;
      }
    return s;
  }
};

// Any settings: the cut, then the draw over the whole row.
template <typename R>
__device__ __noinline__ void sample_many(R row, const Weight weight, bool greedy, int top_k,
                                         float top_p, float min_p, uint32_t u, long long r,
                                         const SampleOut out) {
  Shared& sh = row.sh;
  Cut cut{0u, 0x7fffffff};
  const Steps bin{weight.m, weight.c * (kBins / 32)};
  const float least = weight.below(0x1p-31f);
  if (greedy) {
    cut = cut_top_k(row, 1);
  } else {
    if (top_k > 0 && top_k < row.V)
      cut = cut_by_steps(row, cut, bin, least, least, [&](float x) { return weight(x) != 0 ? 1u : 0u; },
                         NeedCount{(unsigned long long)top_k});
    if (top_p < 1.f) {
      cut = cut_by_steps(row, cut, bin, least, cut.key == 0 ? weight.below(0x1p-16f) : least, weight,
                         NeedMass{fmax(double(top_p), 0.0), 0.0});
    }
  }
  const bool all = cut.key == 0;
  Mass<typename R::E> mass{weight, all ? kNegInf : key_value(cut.key), all ? 0x7fffffff : cut.last, min_p, 0};
  const Found f = find_unit(
      row, fmaxf(fmaxf(least, mass.edge), min_p > 0.f ? weight.below(min_p) : kNegInf), mass,
      [&](unsigned long long total) { return __umul64hi((unsigned long long)u << 32, total) + 1; });
  // the number of tokens kept, if anyone asks
  if (out.n_kept != nullptr) {
    const int n = int(warp_reduce(f.count, AddOp()));
    row.to_all(&sh.frec[row.record()], make_float2(__int_as_float(n), 0.f));
    row.sync();
  }
  if (row.rank == 0 && row.warp == 0) {
    int n = 0;
    if (out.n_kept != nullptr)
      for (int i = row.lane; i < row.records(); i += 32) n += __float_as_int(sh.frec[i].x);
    n = warp_reduce(n, AddOp());
    if (row.lane == 0) out.put(r, f.id, float(double(f.weight) / double(f.total)), n);
  }
}

template <typename R>
ALR_DEV void sample_row(R& row, const SampleArgs& a, const SampleOut& out, long long r) {
  Shared& sh = row.sh;
  const float T = a.temperature != nullptr ? a.temperature[r] : 1.f;
  const int top_k = a.top_k != nullptr ? a.top_k[r] : 0;
  float top_p = a.top_p != nullptr ? a.top_p[r] : 1.f, min_p = a.min_p != nullptr ? a.min_p[r] : 0.f;
  if (!(top_p < 1.f)) top_p = 1.f;   // (NaN too)
  min_p = min_p > 0.f ? fminf(min_p, 1.f) : 0.f;
  const uint32_t u = a.u[r];
  // (a scale that overflows would make the largest token's weight 0 * inf: T = 0 is its limit)
  const float scale = __fdiv_rn(kLog2e, T);
  const bool greedy = !(T > 0.f) || scale == -kNegInf;
  const int K = greedy ? 1 : top_k > 0 && top_k <= kTopMost ? top_k : 0;   // few tokens
  const Bound bound = K > 0 ? bound_and_collect(row, K) : row_bound(row, 0);
  if (!(bound.top > kNegInf)) {   // no candidate; all blocks agree, and none reads another's memory
    if (row.rank == 0 && threadIdx.x == 0) out.put(r, -1, 0.f, 0);
    return;
  }
  const bool infinite = bound.top == -kNegInf;
  const Weight weight{infinite ? 0.f : bound.top, greedy ? 0.f : scale};
  if (K > 0 && (!infinite || K == 1)) {   // (with K = 1 only +inf reaches the bound)
    if (candidates_fit(row)) {
      if (row.rank != 0) return;
      const int n = sort_candidates(row);
      if (!greedy)
        draw_from_candidates(sh, min(n, K), weight, top_p, min_p, u, r, out);
      else if (threadIdx.x == 0)
        out.put(r, entry_id(sh.few.all[0]), 1.f, 1);
      others_know(row);
      return;
    }
  }
  if (infinite) row.only_infinite();
  sample_many(row, weight, greedy, top_k, top_p, min_p, u, r, out);
}

template <typename E, int kPacks>
__global__ void __launch_bounds__(kRowThreadsMost, kPacks > 10 ? 1 : 2)
    sample_kernel(const E* Z, long long ldz, int V, SampleArgs a, SampleOut out, int cluster) {
  __shared__ Shared sh;
  pdl_wait_and_release();
  const long long r = cluster_id_x();
  Row<E, kPacks> row(Z + r * ldz, r * ldz, V, cluster, sh);
  sample_row(row, a, out, r);
}

template <typename E>
__global__ void __launch_bounds__(kStreamThreads, 2)
    sample_stream_kernel(const E* Z, long long N, long long ldz, int V, SampleArgs a, SampleOut out) {
  __shared__ Shared sh;
  pdl_wait_and_release();
  for (long long r = blockIdx.x; r < N; r += gridDim.x) {
    StreamRow<E> row(Z + r * ldz, r * ldz, V, sh);
    sample_row(row, a, out, r);
  }
}

// One block reads a row by itself where there are rows for every SM and a row has a pack for each second
// thread at least.  Streamed and in clusters, us, for [tokens of top-k and top-p; a nucleus; top 64]: 152 rows of
// 151936 bf16 [20, 66, 40] and [103, 115, 70], 768 [82, 250, 168] and [164, 438, 285]; 152 of 32000 fp32 [12, 35,
// 16] and [28, 41, 27]; 152 of 8192 bf16 [10, 30, 13] and [14, 25, 19]; 152 of 2048 bf16 [9, 30, 16] and [40, 21,
// 34].  A nucleus of rows up to 8192 is the cluster's (768 of 2048: 89 and 45), but the settings are on the device.
bool stream_rows(long long N, int V, int sms) { return N >= sms && V >= 2048; }

}  // namespace

cudaError_t launch_top_logits(int dtype, const void* Z, long long N, int V, long long ldz, int K,
                              float t, float* top_val, int32_t* top_idx, float* lse,
                              float* lse_rest, int sms, cudaStream_t s) {
  const TopOut out{top_val, top_idx, lse, lse_rest};
  const auto run = [&](auto* z) {
    using E = std::remove_cv_t<std::remove_pointer_t<decltype(z)>>;
    if (stream_rows(N, V, sms))
      return launch_pdl(top_logits_stream_kernel<E>, dim3(unsigned(std::min<long long>(N, 1 << 20))),
                        dim3(kStreamThreads), 0, s, z, N, ldz, V, K, t, out);
    const RowShape shape = row_shape(N, V, int(sizeof(E)), sms, 256);
    return with_packs(shape.packs, [&](auto packs) {
      return launch_row_each(shape, N, top_logits_kernel<E, decltype(packs)::value>, s, z, ldz, V, K,
                             t, out, shape.cluster);
    });
  };
  return dtype == 0 ? run(static_cast<const __nv_bfloat16*>(Z)) : run(static_cast<const float*>(Z));
}

cudaError_t launch_sample(int dtype, const void* Z, long long N, int V, long long ldz,
                          const SampleArgs& a, int32_t* token, float* prob, int32_t* n_kept, int sms,
                          cudaStream_t s) {
  const SampleOut out{token, prob, n_kept};
  const auto run = [&](auto* z) {
    using E = std::remove_cv_t<std::remove_pointer_t<decltype(z)>>;
    if (stream_rows(N, V, sms))
      return launch_pdl(sample_stream_kernel<E>, dim3(unsigned(std::min<long long>(N, 1 << 20))),
                        dim3(kStreamThreads), 0, s, z, N, ldz, V, a, out);
    const RowShape shape = row_shape(N, V, int(sizeof(E)), sms, 256);
    return with_packs(shape.packs, [&](auto packs) {
      return launch_row_each(shape, N, sample_kernel<E, decltype(packs)::value>, s, z, ldz, V, a, out,
                             shape.cluster);
    });
  };
  return dtype == 0 ? run(static_cast<const __nv_bfloat16*>(Z)) : run(static_cast<const float*>(Z));
}

}  // namespace alr
