// Distillation from a teacher's top logits: the loss of student logits in hand, and its gradient.
//
// Label of a row: softmax over the teacher's listed logits t_i / T and, when given, the log-sum-exp
// of the tokens that are not listed (one bin for all of them).  With s = z / T, m = max s,
// S = sum exp(s - m), R = log-sum-exp of s over the tokens not listed:
//   l = log S + sum_i p_i (m - s_i) + p_0 (m - R)        (no large numbers cancel)
//   dl / dz_v = (q_v - p_v) / T for a listed v, else exp(s_v - R) (q_0 - p_0) / T,
// with q = exp(s) / sum and q_0 the mass outside the list; both factors of the second form are at most 1.
// A bit for each listed token, in shared memory, keeps it out of R's sum, which is taken from the
// largest logit outside the list: exact however small the mass there is (taking the listed terms
// off the whole sum would leave rounding errors of the size of the list's own).  Differences of
// logits are taken before the division by T: they are exact for neighbours.
//
// A row is read once, into the registers of a cluster (row_cluster.cuh), its sums are exchanged between all
// warps once, and the gradient is formed from the same registers.  Clusters stay and take rows in turn: while
// a row is worked on, the next one comes into shared memory, fetched by a warp of its own that reads its
// label too.  2048 x 151936 bf16 logits with 40 % of the rows masked: 228 us, 4.4 TB/s, 0.64 of the copy rate;
// the gradient alone, whose blocks wait for nobody, 4.45 TB/s on rows of two alignments (2000 x 60001).  What is
// left is the blocks' waits for one another's sums (a third of a row's 17 K cycles).  Tried and slower, against
// 215 us when exponentials were of one fma (see exp2_from): one row a cluster, loads straight into registers
// (250: all blocks load, compute and store in step, and memory idles while they compute); the sums of the next
// row taken before the last one's gradient, so that nobody waits (280 with both rows in registers and one block
// to an SM, 293 with rows over 8 blocks); the next row brought into L2 only (no change).
#include "kernels.h"
#include "launch.h"
#include "row_cluster.cuh"

namespace alr {
namespace {

enum { kFwd = 1, kGrad = 2 };

// The row's label in a block's shared memory.
struct Label {
  int idx[kTopMost];       // token, -1 for an absent entry
  float p[kTopMost];       // probability
  float z[kTopMost];       // the student's logit
  float p0, ent;           // the tail bin's probability; entropy
  float z_max, z_sum;      // of the listed tokens' logits (all_z): largest, sum of exponentials from it
  int has;                 // some probability is positive
  long long row;           // the row (N: there is no further one) and its weight
  float w;
};

// One warp reads the row's label, with the student's logits of all listed tokens (all_z) or of those
// in the block's range, whose bits it sets in `listed` (a byte for each pack, from pack `base` on).
template <typename E>
ALR_DEV void read_label(const E* row, const float* val, const int32_t* tok, const float* rest,
                        const DistillArgs& a, bool all_z, int base, int n_packs, int off,
                        uint32_t* listed, Label& l) {
  const int lane = threadIdx.x & 31;
  constexpr int kMost = kTopMost / 32;
  float x[kMost];
  float tm = kNegInf;
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
    const int i = k * 32 + lane;
    x[k] = kNegInf;
    if (k * 32 >= a.K) continue;
    int v = i < a.K ? tok[i] : -1;
    if (v < 0 || v >= a.V) v = -1;
    if (v >= 0) {
      x[k] = val[i];
      const int e = v + off, pack = e / kPerPack<E> - base;
      const bool here = pack >= 0 && pack < n_packs;
      if (here || all_z) l.z[i] = to_float(row[v]);
      if (here) atomicOr(&listed[pack >> 2], 1u << ((pack & 3) * 8 + e % kPerPack<E>));
    }
    if (i < a.K) l.idx[i] = v;
    tm = fmaxf(tm, x[k]);
  }
  tm = warp_max(tm);
  // The larger of the list's first and the bin leads; m may leave a float's range (the type's lowest value
  // by T < 1) though the list has its softmax, so not m but its parts say whether there is a label.
  const float x0 = rest != nullptr ? *rest : kNegInf, tl = tm * a.inv_t, m = fmaxf(tl, x0);
  const bool has = tm > kNegInf || x0 > kNegInf;
  const float step = x0 > tl ? tl - x0 : 0.f;   // 0 unless the bin leads
  const float d0 = x0 - m, e0 = d0 > kNegInf ? expf(d0) : 0.f;   // (-inf - -inf: no bin)
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
    if (k * 32 >= a.K) break;
    x[k] = x[k] > kNegInf ? (x[k] - tm) * a.inv_t + step : kNegInf;
    sum += x[k] > kNegInf ? expf(x[k]) : 0.f;
  }
  sum = warp_reduce(sum, AddOp()) + (has ? e0 : 0.f);
  const float ls = logf(sum), inv = has ? 1.f / sum : 0.f;
  float h = 0.f;
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
    const int i = k * 32 + lane;
    if (i >= a.K) break;
    const float p = x[k] > kNegInf ? expf(x[k]) * inv : 0.f;
    l.p[i] = p;
    if (p > 0.f) h += p * (ls - x[k]);
  }
  h = warp_reduce(h, AddOp());
  if (lane == 0) {
    const float p0 = has ? e0 * inv : 0.f;
    l.p0 = p0;
    l.has = has;
    l.ent = p0 > 0.f ? h + p0 * (ls - d0) : h;
  }
  if (all_z) {
    __syncwarp();
    float zm = kNegInf, zs = 0.f;
    for (int i = lane; i < a.K; i += 32)
      if (l.idx[i] >= 0) zm = fmaxf(zm, l.z[i]);
    zm = warp_max(zm);
    if (zm > kNegInf)
      for (int i = lane; i < a.K; i += 32)
        if (l.idx[i] >= 0) zs += expf((l.z[i] - zm) * a.inv_t);
    zs = warp_reduce(zs, AddOp());
    if (lane == 0) {
      l.z_max = zm;
      l.z_sum = zs;
    }
  }
}

ALR_DEV uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// exp2((x - ref) k) of two elements.  The difference first: one fma, x k - ref k, would carry the rounding of
// ref k, which for logits / T past 2^30 (a mask by a large finite number over a whole stretch of the row, a
// tiny T) is out of the exponential's range, and of a float's for the type's lowest value: NaN.  (It was 223 us
// instead of 229 for loss and gradient of the rows above, nothing for either alone.)
ALR_DEV uint64_t exp2_from(uint64_t x, uint64_t ref, uint64_t k) {
  return f2_ex2(f2_mul(f2_sub(x, ref), k));
}

// Gradient of a pack, c exp2((x - ref) k), in the row's element type.
template <typename E>
ALR_DEV uint4 grad_pack(const uint4& raw, float ref, float k, float c) {
  float q[kPerPack<E>];
  const uint64_t ref2 = f2_pack(ref, ref), k2 = f2_pack(k, k), c2 = f2_pack(c, c);
#pragma unroll
  for (int e = 0; e < kPerPack<E>; e += 2) {
    const uint64_t x = f2_pack(pack_elem<E>(raw, e), pack_elem<E>(raw, e + 1));
    f2_unpack(f2_mul(exp2_from(x, ref2, k2), c2), q[e], q[e + 1]);
  }
  if constexpr (sizeof(E) == 2)
    return make_uint4(pack_bf16(q[0], q[1]), pack_bf16(q[2], q[3]), pack_bf16(q[4], q[5]),
                      pack_bf16(q[6], q[7]));
  else
    return make_uint4(__float_as_uint(q[0]), __float_as_uint(q[1]), __float_as_uint(q[2]),
                      __float_as_uint(q[3]));
}

// A pack of results to the row's elements [v, v + kPerPack), those within [lo, hi).
template <typename E>
ALR_DEV void store_elems(E* g, int v, int lo, int hi, const uint4& x) {
#pragma unroll
  for (int e = 0; e < kPerPack<E>; ++e)
    if (v + e >= lo && v + e < hi) g[v + e] = E(pack_elem<E>(x, e));
}

template <typename E>
ALR_DEV void store_pack(E* g, int v, int V, const uint4& x) {
  if (v >= 0 && v + kPerPack<E> <= V)
    __stcs(reinterpret_cast<uint4*>(g + v), x);
  else
    store_elems(g, v, 0, V, x);
}

// A warp's consecutive packs to a row whose 16-byte boundaries lie `shift` elements (1 .. kPerPack - 1)
// before theirs: what goes into one there is the end of one pack and the start of the next.  Called for
// the thread's packs i in order; `prev`: the thread's pack i - 1.
template <typename E>
ALR_DEV void store_shifted(E* g, int v, int V, int shift, bool first, bool last, const uint4& prev,
                           const uint4& x) {
  const int lane = threadIdx.x & 31, bytes = shift * int(sizeof(E));
  // the pack before this one: the lane below's, or the last lane's of the row of packs before
  const uint32_t own[4] = {x.x, x.y, x.z, x.w};
  const uint32_t old[4] = {prev.x, prev.y, prev.z, prev.w};
  uint32_t c[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    c[j] = __shfl_sync(0xffffffffu, lane == 31 ? old[j] : own[j], (lane + 31) & 31);
    c[j + 4] = own[j];
  }
  // the 16 bytes of c that start 16 - bytes in
  const int from = 3 - (bytes >> 2);
  uint32_t b[6], s[5];
#pragma unroll
  for (int j = 0; j < 6; ++j) b[j] = from & 2 ? c[j + 2] : c[j];
#pragma unroll
  for (int j = 0; j < 5; ++j) s[j] = from & 1 ? b[j + 1] : b[j];
  const uint32_t pick = bytes & 2 ? 0x5432u : 0x7654u;
  const uint4 o = make_uint4(__byte_perm(s[0], s[1], pick), __byte_perm(s[1], s[2], pick),
                             __byte_perm(s[2], s[3], pick), __byte_perm(s[3], s[4], pick));
  const int at = v - shift;
  if (first && lane == 0)   // the end of another warp's pack is that warp's
    store_elems(g, v, 0, min(V, v + kPerPack<E> - shift), x);
  else if (at >= 0 && at + kPerPack<E> <= V)
    __stcs(reinterpret_cast<uint4*>(g + at), o);
  else
    store_elems(g, at, 0, V, o);
  if (last && lane == 31) store_elems(g, v, max(0, v + kPerPack<E> - shift), V, x);
}

// What a block's first warp makes of the cluster's records, for all of its warps.
struct RowSums {
  float ref, b;         // log2 q_v = (z_v - ref) k + b
  float out_ref, out_c; // gradient outside the list: out_c exp2((z_v - out_ref) k)
  float c;              // lambda w / (T sum w); 0 when the row has no gradient
  float top;            // the largest logit if some token outside the list has it, else NaN
  int writer;           // the cluster's warp that writes the greedy token
};

// exp(x / T - lse) = 2^((x - ref) k + log_scale) with ref a logit next to T lse: the products then are of
// small numbers, and what ref leaves of lse is the scale.  (exp2(x k - lse log2 e) loses 2^-24 |lse| on the
// way, up to half as much again as lse's own rounding costs.)
// q is off by 2^-24 |lse| relative, the rounding of lse itself.  From kLseMost on that says nothing (an lse of
// tokens masked by large finite numbers alone, a tiny T): the gradient is 0 there.
constexpr float kLseMost = 16777216.f;
struct FromLse {
  float ref, log_scale;
};
ALR_DEV FromLse from_lse(float lse, float t, float k) {
  const float ref = lse * t;
  return {ref, fmaf(-lse, t, ref) * k};
}

// Named barriers: the row's data and label are there; the data is in registers (of the fetching warp
// and the others); the sums are there; the gradient outside the list is written (of the others).
enum { kBarFull = 1, kBarTaken, kBarSums, kBarWritten };

template <typename E, int kPacks>
struct RowBuffer {   // dynamic shared memory: a slice of a row, then `listed` of two rows
  uint4* data;
  uint8_t* listed;
  int n_packs;
  ALR_DEV RowBuffer(unsigned char* smem, int threads)
      : data(reinterpret_cast<uint4*>(smem)),
        listed(smem + size_t(threads) * kPacks * 16),
        n_packs(threads * kPacks) {}
  static size_t bytes(int threads) { return size_t(threads) * kPacks * 18; }
};

// Blocks of T threads that work on rows and a warp that fetches them; cluster i of n takes the rows i,
// i + n, ...  kFwd: a row's loss, entropy, log-sum-exps and greedy token; kGrad: the gradient of its
// logits, from this row's sums or (kGrad alone) from lse, lse_rest of a forward.  A wait that runs out
// is recorded and the kernel goes on to its end with what it has.
template <typename E, int kPacks, int kMode>
__global__ void __launch_bounds__(kRowThreadsMost + 32, kPacks > 10 ? 1 : 2)
    distill_row_kernel(const E* Z, const float* top_val, const int32_t* top_idx, const float* rest,
                       const float* weight, const float* norm, DistillArgs a, DistillRows o,
                       float* weight_sum, E* G, int cluster, int* status) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ Label labels[2];
  __shared__ RowSums row_sums[2];
  // of each warp of the cluster: largest logit outside the list, sum of exponentials from it
  __shared__ float2 recs[2][kRowWarpsMost * kRowClusterMost];
  __shared__ uint64_t full_bar, rec_bar[2];
  __shared__ double wbuf[32];
  __shared__ volatile int abort_word;
  const int threads = int(blockDim.x) - 32, n_warps = threads / 32;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
  const int rank = int(cluster_ctarank()), first_row = int(cluster_id_x()), step = int(n_clusters_x());
  const RowBuffer<E, kPacks> buf(smem, threads);
  const AbortFlag ab{&abort_word, status};
  const bool fetcher = warp == n_warps;
  if (tid == 0) {
    abort_word = 0;
    mbar_init(&full_bar, 1);
    mbar_init(&rec_bar[0], 1);
    mbar_init(&rec_bar[1], 1);
    fence_mbar_init();
  }
  pdl_wait_and_release();
  if constexpr ((kMode & kFwd) != 0)
    cluster_sync();   // the peers' barriers are there
  else
    __syncthreads();

  const auto next_live = [&](long long r) {   // rows of weight 0 are not read
    while (r < a.N && weight != nullptr && weight[r] == 0.f) r += step;
    return r;
  };
  // The block's part of row r, whole packs of it, into the buffer.
  const auto fetch = [&](long long r) {
    if (lane != 0) return;
    const RowPlace<E, kPacks> at(r * a.ldz, rank, threads);
    const int lo = max(at.base, at.off > 0 ? 1 : 0);
    const int hi = min(at.base + buf.n_packs, (a.V + at.off) / kPerPack<E>);
    if (hi > lo) {
      fence_proxy_async_smem();
      const uint32_t bytes = uint32_t(hi - lo) * 16;
      mbar_arrive_expect_tx(&full_bar, bytes);
      bulk_load(smem_u32(buf.data + (lo - at.base)), Z + r * a.ldz + (lo * kPerPack<E> - at.off), bytes,
                &full_bar);
    } else {
      mbar_arrive(&full_bar);
    }
  };
  long long live = 0;   // fetching warp: the row that it fetches
  if (fetcher) {
    live = next_live(first_row);
    if (live < a.N) fetch(live);
  }
  // sum w, in the same order in every block
  float wsum = float(a.N);
  if (weight != nullptr &&
      ((kMode & kGrad) && norm == nullptr || (kMode & kFwd) && blockIdx.x == 0)) {
    double s = 0.0;
#pragma unroll 8
    for (long long r = tid; r < a.N; r += blockDim.x) s += double(weight[r]);
    wsum = float(block_reduce(s, AddOp(), wbuf));
  }
  if ((kMode & kFwd) && blockIdx.x == 0 && tid == 0) *weight_sum = wsum;
  const float ws = norm != nullptr ? *norm : wsum;

  if (fetcher) {
    for (uint32_t n = 0;; ++n) {
      const long long r = live;
      Label& lab = labels[n & 1];
      if (n > 0) {
        named_bar_sync(kBarTaken, threads + 32);
        if (r < a.N) fetch(r);
      }
      if (lane == 0) {
        lab.row = r;
        if (r < a.N) lab.w = weight != nullptr ? weight[r] : 1.f;
      }
      if (r >= a.N) {
        __syncwarp();
        named_bar_arrive(kBarFull, threads + 32);
        break;
      }
      const E* z = Z + r * a.ldz;
      const RowPlace<E, kPacks> at(r * a.ldz, rank, threads);
      // a first and a last pack that are the row's in part
      if (lane < 2) {
        const int pack = lane == 0 ? 0 : (a.V + at.off) / kPerPack<E>;
        const int v = pack * kPerPack<E> - at.off;
        const bool part = lane == 0 ? at.off > 0 : v < a.V && (v >= 0 || at.off == 0);
        if (part && pack >= at.base && pack < at.base + buf.n_packs)
          buf.data[pack - at.base] = load_pack(z, v, a.V);
      }
      uint32_t* listed = reinterpret_cast<uint32_t*>(buf.listed + (n & 1) * buf.n_packs);
      for (int i = lane; i < buf.n_packs / 4; i += 32) listed[i] = 0;
      __syncwarp();
      read_label(z, top_val + r * a.K, top_idx + r * a.K, rest != nullptr ? rest + r : nullptr, a,
                 (kMode & kFwd) != 0, at.base, buf.n_packs, at.off, listed, lab);
      live = next_live(r + step);
      mbar_wait(&full_bar, n & 1, ab);
      __syncwarp();
      named_bar_arrive(kBarFull, threads + 32);
    }
  } else {
    const float k = a.inv_t * kLog2e;
    long long next = first_row;
    for (uint32_t n = 0;; ++n) {
      const uint32_t par = n & 1, phase = (n >> 1) & 1;
      const Label& lab = labels[par];
      named_bar_sync(kBarFull, threads + 32);
      const long long r = lab.row;
      for (; next < r && next < a.N; next += step) {   // rows of weight 0
        if ((kMode & kFwd) && rank == 0 && tid == 0) {
          o.loss_row[next] = 0.f;
          if (o.ent_row != nullptr) o.ent_row[next] = 0.f;
          o.lse[next] = 0.f;
          if (o.lse_rest != nullptr) o.lse_rest[next] = 0.f;
          if (o.argmax != nullptr) o.argmax[next] = -1;
        }
        if constexpr ((kMode & kGrad) != 0) {
          const RowPlace<E, kPacks> to(next * a.ldg, rank, threads);
#pragma unroll
          for (int i = 0; i < kPacks; ++i)
            store_pack(G + next * a.ldg, to.elem(i), a.V, make_uint4(0, 0, 0, 0));
        }
      }
      if (r >= a.N) break;
      next = r + step;
      E* g = G + r * a.ldg;
      RowSums& sums = row_sums[par];
      const RowPlace<E, kPacks> at(r * a.ldz, rank, threads);
      const int local = at.pack - at.base;
      const uint8_t* listed = buf.listed + par * buf.n_packs + local;
      const bool whole = at.whole(a.V);
      uint4 raw[kPacks];
#pragma unroll
      for (int i = 0; i < kPacks; ++i) {
        raw[i] = buf.data[local + 32 * i];
        if (!whole) {
          const int v = at.elem(i);
          if (v >= a.V || v + kPerPack<E> <= 0) raw[i] = neg_inf_pack<E>();
        }
      }
      named_bar_arrive(kBarTaken, threads + 32);
      if constexpr ((kMode & kFwd) != 0) {
        float m = kNegInf;
#pragma unroll
        for (int i = 0; i < kPacks; ++i) {
          mask_pack<E>(raw[i], listed[32 * i]);   // the listed tokens are handled apart from here on
#pragma unroll
          for (int e = 0; e < kPerPack<E>; e += 2)
            m = max3(m, pack_elem<E>(raw[i], e), pack_elem<E>(raw[i], e + 1));
        }
        m = warp_max(m);
        const float mw = m > kNegInf ? m : 0.f;
        const uint64_t ref2 = f2_pack(mw, mw), k2 = f2_pack(k, k);
        uint64_t s2 = 0;
#pragma unroll
        for (int i = 0; i < kPacks; ++i)
#pragma unroll
          for (int e = 0; e < kPerPack<E>; e += 2) {
            const uint64_t x = f2_pack(pack_elem<E>(raw[i], e), pack_elem<E>(raw[i], e + 1));
            s2 = f2_add(s2, exp2_from(x, ref2, k2));
          }
        float sa, sb;
        f2_unpack(s2, sa, sb);
        const float sw = warp_reduce(sa + sb, AddOp());
        if (lane < cluster)   // to every block of the cluster
          st_async_f2(cluster_smem_addr(&recs[par][rank * n_warps + warp], lane), m, sw,
                      cluster_smem_addr(&rec_bar[par], lane));
      }
      // The first warp makes the row's sums of the records; what the others wait for comes first.
      float ls = 0.f, lo = 0.f, gap = 0.f, mt = 0.f;
      bool any = false, some = false;
      if (warp == 0) {
        float c = lab.has && ws > 0.f ? a.lambda * lab.w / ws * a.inv_t : 0.f;
        if constexpr ((kMode & kFwd) != 0) {
          const int n_rec = n_warps * cluster;
          if (lane == 0) mbar_arrive_expect_tx(&rec_bar[par], uint32_t(n_rec) * 8);
          const float zl = lab.z_max;
          __syncwarp();
          mbar_wait_cluster(&rec_bar[par], phase, ab);
          constexpr int kMost = kRowWarpsMost * kRowClusterMost / 32 + 1;
          float mo = kNegInf, So = 0.f;
          float2 t[kMost];
#pragma unroll
          for (int j = 0; j < kMost; ++j) {
            t[j] = make_float2(kNegInf, 0.f);
            if (j * 32 + lane < n_rec) t[j] = recs[par][j * 32 + lane];
            mo = fmaxf(mo, t[j].x);
          }
          mo = warp_max(mo);
          int first = 0x7fffffff;
#pragma unroll
          for (int j = kMost - 1; j >= 0; --j) {
            if (!(t[j].x > kNegInf)) continue;
            So += t[j].y * ex2((t[j].x - mo) * k);
            if (t[j].x == mo) first = j * 32 + lane;
          }
          So = warp_reduce(So, AddOp());
          first = warp_min(first);   // the warp with the first of the largest, if any
          any = mo > kNegInf;
          const float top = fmaxf(mo, zl);
          some = top > kNegInf;
          mt = some ? top : 0.f;
          gap = (mo - mt) * a.inv_t;   // -inf when everything is listed
          const float So_t = any ? So * expf(gap) : 0.f;
          const float S = So_t + (zl > kNegInf ? lab.z_sum * expf((zl - mt) * a.inv_t) : 0.f);
          ls = logf(S);
          lo = logf(So);
          if (lane == 0) {
            if (!some) c = 0.f;
            sums.c = c;
            sums.ref = mt;
            sums.b = -ls * kLog2e;
            sums.out_ref = any ? mo : 0.f;
            sums.out_c = any ? c * (So_t / S - lab.p0) / So : 0.f;
            // the greedy token is written by the warp that holds the first of the largest logits
            // outside the list, or by the first warp when the list holds all of them
            sums.top = mo == top && any ? top : __builtin_nanf("");
            sums.writer = mo == top && any ? first : 0;
            if (rank == 0) {
              o.lse[r] = mt / a.t + ls;
              if (o.lse_rest != nullptr) o.lse_rest[r] = any ? mo / a.t + lo : kNegInf;
            }
          }
        } else if (lane == 0) {
          const float lse = o.lse[r], lse_rest = rest != nullptr ? o.lse_rest[r] : kNegInf;
          const bool known = fabsf(lse) < kLseMost, rest_known = fabsf(lse_rest) < kLseMost;
          if (!known) c = 0.f;
          sums.c = c;
          const FromLse q = from_lse(known ? lse : 0.f, a.t, k);
          sums.ref = q.ref;
          sums.b = q.log_scale;
          if (rest == nullptr) {
            sums.out_ref = q.ref;
            sums.out_c = c * ex2(q.log_scale);
          } else {
            const FromLse o = from_lse(rest_known ? lse_rest : 0.f, a.t, k);
            sums.out_ref = rest_known ? o.ref : -kNegInf;   // from there every exponential is 0
            sums.out_c = rest_known ? c * (expf(lse_rest - lse) - lab.p0) * ex2(o.log_scale) : 0.f;
          }
        }
      }
      named_bar_sync(kBarSums, threads);
      if constexpr ((kMode & kFwd) != 0) {
        if (rank == 0 && warp == 0) {
          float loss = 0.f;
          for (int i = lane; i < a.K; i += 32)
            if (lab.p[i] > 0.f) loss += lab.p[i] * (ls + (mt - lab.z[i]) * a.inv_t);
          loss = warp_reduce(loss, AddOp());
          if (lab.p0 > 0.f) loss += lab.p0 * (ls - (lo + gap));
          if (lane == 0) {
            const bool on = lab.has && some;
            o.loss_row[r] = on ? loss : 0.f;
            if (o.ent_row != nullptr) o.ent_row[r] = on ? lab.ent : 0.f;
          }
        }
        if (o.argmax != nullptr && rank * n_warps + warp == sums.writer) {
          float best = sums.top;   // NaN: no token outside the list has the largest logit
          int v = 0x7fffffff;
          if (best == best) {
#pragma unroll
            for (int i = 0; i < kPacks; ++i)
#pragma unroll
              for (int e = 0; e < kPerPack<E>; ++e)
                if (pack_elem<E>(raw[i], e) == best) v = min(v, at.elem(i) + e);
          } else {
            best = lab.z_max;
          }
          for (int i = lane; i < a.K; i += 32)
            if (lab.idx[i] >= 0 && lab.z[i] == best) v = min(v, lab.idx[i]);
          v = warp_min(v);
          if (lane == 0) o.argmax[r] = best > kNegInf ? v : -1;
        }
      }
      if constexpr ((kMode & kGrad) != 0) {
        const float c = sums.c, out_ref = sums.out_ref, out_c = sums.out_c;
        if (c == 0.f) {
#pragma unroll
          for (int i = 0; i < kPacks; ++i) raw[i] = neg_inf_pack<E>();
        }
        if (int(r * a.ldg % kPerPack<E>) == at.off) {
          if (whole) {
            uint4* p = reinterpret_cast<uint4*>(g + at.elem(0));
#pragma unroll
            for (int i = 0; i < kPacks; ++i)
              __stcs(p + 32 * i, grad_pack<E>(raw[i], out_ref, k, out_c));
          } else {
#pragma unroll
            for (int i = 0; i < kPacks; ++i)
              store_pack(g, at.elem(i), a.V, grad_pack<E>(raw[i], out_ref, k, out_c));
          }
        } else {
          const int shift =
              (int(r * a.ldg % kPerPack<E>) - at.off + kPerPack<E>) % kPerPack<E>;
          uint4 prev = make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < kPacks; ++i) {
            const uint4 x = grad_pack<E>(raw[i], out_ref, k, out_c);
            store_shifted(g, at.elem(i), a.V, shift, i == 0, i == kPacks - 1, prev, x);
            prev = x;
          }
        }
        // over them, the listed tokens of this block's range
        named_bar_sync(kBarWritten, threads);
        for (int i = tid; i < a.K; i += threads) {
          const int v = lab.idx[i], pack = (v + at.off) / kPerPack<E> - at.base;
          if (v >= 0 && pack >= 0 && pack < buf.n_packs)
            g[v] = E(c != 0.f ? c * (ex2(fmaf(lab.z[i] - sums.ref, k, sums.b)) - lab.p[i]) : 0.f);
        }
      }
    }
  }
  if constexpr ((kMode & kFwd) != 0) cluster_sync();   // until no block writes into this one's records
}

// L = lambda sum w l / sum w, one block, fixed order.
__global__ void __launch_bounds__(1024)
    distill_loss_kernel(const float* weight, const float* loss_row, float* weight_sum, long long N,
                        float lambda, float* loss_total, float* wl_sum) {
  __shared__ double buf[32];
  pdl_wait_and_release();
  double s = 0.0;
  for (long long r = threadIdx.x; r < N; r += 1024)
    s += double(loss_row[r]) * (weight != nullptr ? double(weight[r]) : 1.0);
  s = block_reduce(s, AddOp(), buf);
  if (threadIdx.x == 0) {
    if (N == 0) *weight_sum = 0.f;
    const double ws = *weight_sum;
    *loss_total = ws > 0.0 ? float(double(lambda) * s / ws) : 0.f;
    if (wl_sum != nullptr) *wl_sum = float(s);
  }
}

template <typename E, int kPacks>
cudaError_t launch_rows(const RowShape& shape, const DistillArgs& a, bool fwd, bool grad,
                        const void* Z, const float* top_val, const int32_t* top_idx,
                        const float* rest, const float* weight, const float* norm,
                        const DistillRows& o, float* weight_sum, void* G, int sms, int* status,
                        cudaStream_t s) {
  auto kern = fwd ? (grad ? distill_row_kernel<E, kPacks, kFwd | kGrad>
                          : distill_row_kernel<E, kPacks, kFwd>)
                  : distill_row_kernel<E, kPacks, kGrad>;
  return launch_row_clusters(shape, shape.threads + 32, RowBuffer<E, kPacks>::bytes(shape.threads),
                             a.N, sms, kern, s, static_cast<const E*>(Z), top_val, top_idx, rest,
                             weight, norm, a, o, weight_sum, static_cast<E*>(G), shape.cluster,
                             status);
}

}  // namespace

cudaError_t launch_distill(const DistillArgs& a, bool fwd, bool grad, const void* Z,
                           const float* top_val, const int32_t* top_idx, const float* rest,
                           const float* weight, const float* norm, const DistillRows& o,
                           const DistillSums& t, void* G, int sms, int* status, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  if (a.N > 0) {
    const RowShape shape = row_shape(a.N, a.V, a.dtype == 0 ? 2 : 4, sms);
    e = with_packs(shape.packs, [&](auto packs) {
      constexpr int kP = decltype(packs)::value;
      return a.dtype == 0
                 ? launch_rows<__nv_bfloat16, kP>(shape, a, fwd, grad, Z, top_val, top_idx, rest,
                                                  weight, norm, o, t.weight_sum, G, sms, status, s)
                 : launch_rows<float, kP>(shape, a, fwd, grad, Z, top_val, top_idx, rest, weight,
                                          norm, o, t.weight_sum, G, sms, status, s);
    });
    if (e != cudaSuccess) return e;
  }
  if (fwd)
    e = launch_pdl(distill_loss_kernel, dim3(1), dim3(1024), 0, s, weight, o.loss_row,
                   t.weight_sum, a.N, a.lambda, t.loss_total, t.wl_sum);
  return e;
}

}  // namespace alr
