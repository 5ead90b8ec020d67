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
// Memory-bound: a row is read once into the registers of a cluster (row_cluster.cuh); its sums are
// exchanged between the warps once, through distributed shared memory, and the gradient is formed from the
// same registers.
#include "kernels.h"
#include "launch.h"
#include "row_cluster.cuh"

namespace alr {
namespace {

enum { kFwd = 1, kGrad = 2 };

// The row's label in a block's shared memory.
struct LabelShared {
  int idx[kTopMost];       // token, -1 for an absent entry
  float p[kTopMost];       // probability
  float z[kTopMost];       // the student's logit
  float p0, ent;           // the tail bin's probability; entropy
  int has;                 // some probability is positive
};

// One warp reads the row's label.  `z` is read for tokens in [lo, hi); the bits of those of
// the block's range are set in `listed` (a byte for each pack, from pack `base` on).
template <typename E>
ALR_DEV void read_label(const E* row, const float* val, const int32_t* tok, const float* rest,
                        const DistillArgs& a, bool all_z, int base, int n_packs, int off,
                        uint32_t* listed, LabelShared& l) {
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
  tm = warp_reduce(tm, MaxOp());
  const float x0 = rest != nullptr ? *rest : kNegInf, m = fmaxf(tm * a.inv_t, x0);
  const bool has = m > kNegInf;
  const float step = tm > kNegInf ? tm * a.inv_t - m : 0.f;   // 0 unless the bin leads
  const float d0 = x0 - m, e0 = d0 > kNegInf ? expf(d0) : 0.f;
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
}

ALR_DEV uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Gradient of a pack, c exp2((x - ref) k + b), in the row's element type; `b` takes ref in.
template <typename E>
ALR_DEV uint4 grad_pack(const uint4& raw, float k, float b, float c) {
  float q[kPerPack<E>];
  const uint64_t k2 = f2_pack(k, k), b2 = f2_pack(b, b), c2 = f2_pack(c, c);
#pragma unroll
  for (int e = 0; e < kPerPack<E>; e += 2) {
    const uint64_t x = f2_pack(pack_elem<E>(raw, e), pack_elem<E>(raw, e + 1));
    f2_unpack(f2_mul(f2_ex2(f2_fma(x, k2, b2)), c2), q[e], q[e + 1]);
  }
  if constexpr (sizeof(E) == 2)
    return make_uint4(pack_bf16(q[0], q[1]), pack_bf16(q[2], q[3]), pack_bf16(q[4], q[5]),
                      pack_bf16(q[6], q[7]));
  else
    return make_uint4(__float_as_uint(q[0]), __float_as_uint(q[1]), __float_as_uint(q[2]),
                      __float_as_uint(q[3]));
}

// A pack of results to the row's elements [v, v + kPerPack) within it, but for those of `skip`.
template <typename E>
ALR_DEV void store_elems(E* g, int v, int V, uint32_t skip, const uint4& x) {
#pragma unroll
  for (int e = 0; e < kPerPack<E>; ++e)
    if (!(skip >> e & 1) && v + e >= 0 && v + e < V) g[v + e] = E(pack_elem<E>(x, e));
}

// What a block's first warp makes of the cluster's records, for all of its warps.
struct RowSums {
  float ref, b;         // log2 q_v = (z_v - ref) k + b
  float out_b, out_c;   // gradient outside the list: out_c exp2(z_v k + out_b)
  float c;              // lambda w / (T sum w); 0 when the row has no gradient
  float top;            // the largest logit if some token outside the list has it, else NaN
  int writer;           // the cluster's warp that writes the greedy token
};

// exp2((x - m) k) with one fma: exp2(x k + b), b = -m k rounded, carries the factor 2^r with
// r = m k + b, the same for every x, which the caller takes off once.
ALR_DEV float ref_offset(float m, float k) { return -m * k; }
ALR_DEV float ref_residual(float m, float k) { return fmaf(m, k, ref_offset(m, k)); }

// One cluster per row.  kFwd: the row's loss, entropy, log-sum-exps and greedy token; kGrad: the
// gradient of its logits, from this row's sums or (kGrad alone) from lse, lse_rest of a forward.
template <typename E, int kPacks, int kMode>
__global__ void __launch_bounds__(kRowThreadsMost, kPacks > 10 ? 1 : 2)
    distill_row_kernel(const E* Z, const float* top_val, const int32_t* top_idx, const float* rest,
                       const float* weight, const float* weight_sum, DistillArgs a,
                       DistillRows o, E* G, int cluster) {
  __shared__ uint32_t listed[kRowThreadsMost * kPacks / 4];
  __shared__ LabelShared lab;
  __shared__ RowSums sums;
  __shared__ float2 rec[kRowWarpsMost];   // of each warp: largest logit outside the list, sum
  pdl_wait_and_release();
  const int rank = cluster > 1 ? int(cluster_ctarank()) : 0;
  const long long r = cluster > 1 ? cluster_id_x() : blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32, n_warps = blockDim.x / 32;
  const E* z = Z + r * a.ldz;
  E* g = G + r * a.ldg;
  const float w = weight != nullptr ? weight[r] : 1.f;
  if (w == 0.f) {   // not read
    if ((kMode & kFwd) && rank == 0 && tid == 0) {
      o.loss_row[r] = 0.f;
      if (o.ent_row != nullptr) o.ent_row[r] = 0.f;
      o.lse[r] = 0.f;
      if (o.lse_rest != nullptr) o.lse_rest[r] = 0.f;
      if (o.argmax != nullptr) o.argmax[r] = -1;
    }
    if constexpr ((kMode & kGrad) != 0) {
      const RowPlace<E, kPacks> to(r * a.ldg, rank);
      const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < kPacks; ++i) {
        const int v = to.elem(i);
        if (v >= 0 && v + kPerPack<E> <= a.V)
          __stcs(reinterpret_cast<uint4*>(g + v), zero);
        else
          store_elems(g, v, a.V, 0, zero);
      }
    }
    return;
  }
  const RowPlace<E, kPacks> at(r * a.ldz, rank);
  uint4 raw[kPacks];
  load_row(raw, z, at, a.V);
  const int n_packs = int(blockDim.x) * kPacks;
  for (int i = tid; i < n_packs / 4; i += blockDim.x) listed[i] = 0;
  __syncthreads();
  if (warp == 0)
    read_label(z, top_val + r * a.K, top_idx + r * a.K, rest != nullptr ? rest + r : nullptr, a,
               (kMode & kFwd) != 0, at.base, n_packs, at.off, listed, lab);
  __syncthreads();
  const uint8_t* listed_bytes = reinterpret_cast<const uint8_t*>(listed) + (at.pack - at.base);
  const float k = a.inv_t * kLog2e;
  if constexpr ((kMode & kFwd) != 0) {
    float m = kNegInf;
#pragma unroll
    for (int i = 0; i < kPacks; ++i) {
      mask_pack<E>(raw[i], listed_bytes[32 * i]);   // the listed tokens are handled apart from here on
#pragma unroll
      for (int e = 0; e < kPerPack<E>; e += 2)
        m = max3(m, pack_elem<E>(raw[i], e), pack_elem<E>(raw[i], e + 1));
    }
    m = warp_reduce(m, MaxOp());
    const float mw = m > kNegInf ? m : 0.f, off = ref_offset(mw, k);
    const uint64_t off2 = f2_pack(off, off), k2 = f2_pack(k, k);
    uint64_t s2 = 0;
#pragma unroll
    for (int i = 0; i < kPacks; ++i)
#pragma unroll
      for (int e = 0; e < kPerPack<E>; e += 2) {
        const uint64_t x = f2_pack(pack_elem<E>(raw[i], e), pack_elem<E>(raw[i], e + 1));
        s2 = f2_add(s2, f2_ex2(f2_fma(x, k2, off2)));
      }
    float sa, sb;
    f2_unpack(s2, sa, sb);
    const float sw = warp_reduce(sa + sb, AddOp()) * ex2(-ref_residual(mw, k));
    if (lane == 0) rec[warp] = make_float2(m, sw);
    if (cluster > 1)
      cluster_sync();
    else
      __syncthreads();
  }
  if (warp == 0) {
    float c = 0.f;
    if constexpr ((kMode & kGrad) != 0) {
      const float ws = *weight_sum;
      c = lab.has && ws > 0.f ? a.lambda * w / ws * a.inv_t : 0.f;
    }
    if constexpr ((kMode & kFwd) != 0) {
      // the records of all warps of the cluster, in the order of the row
      constexpr int kMost = kRowWarpsMost * kRowClusterMost / 32;
      const int n_rec = n_warps * cluster;
      float2 t[kMost];
      float mo = kNegInf;
#pragma unroll
      for (int j = 0; j < kMost; ++j) {
        t[j] = make_float2(kNegInf, 0.f);
        if (j * 32 >= n_rec) continue;
        const int i = j * 32 + lane;
        if (i < n_rec)
          t[j] = cluster > 1 ? ld_cluster_f2(cluster_smem_addr(&rec[i % n_warps], i / n_warps))
                             : rec[i];
        mo = fmaxf(mo, t[j].x);
      }
      mo = warp_reduce(mo, MaxOp());
      float So = 0.f;
      int first = 0x7fffffff;
#pragma unroll
      for (int j = 0; j < kMost; ++j) {
        if (t[j].x > kNegInf) So += t[j].y * ex2((t[j].x - mo) * k);
        if (t[j].x == mo && t[j].x > kNegInf) first = min(first, j * 32 + lane);
      }
      So = warp_reduce(So, AddOp());
      first = warp_reduce(first, MinOp());   // the warp with the first of the largest, if any
      float zl = kNegInf;
      for (int i = lane; i < a.K; i += 32)
        if (lab.idx[i] >= 0) zl = fmaxf(zl, lab.z[i]);
      const float top = fmaxf(mo, warp_reduce(zl, MaxOp())), mt = top > kNegInf ? top : 0.f;
      float S = 0.f;
      for (int i = lane; i < a.K; i += 32)
        if (lab.idx[i] >= 0) S += expf((lab.z[i] - mt) * a.inv_t);
      S = warp_reduce(S, AddOp());
      const float gap = (mo - mt) * a.inv_t;   // -inf when everything is listed
      if (mo > kNegInf) S += So * expf(gap);
      const float ls = logf(S), lo = logf(So);
      if (rank == 0) {
        float loss = 0.f;
        for (int i = lane; i < a.K; i += 32)
          if (lab.p[i] > 0.f) loss += lab.p[i] * (ls + (mt - lab.z[i]) * a.inv_t);
        loss = warp_reduce(loss, AddOp());
        if (lab.p0 > 0.f) loss += lab.p0 * (ls - (lo + gap));
        if (lane == 0) {
          const bool on = lab.has && top > kNegInf;
          o.loss_row[r] = on ? loss : 0.f;
          if (o.ent_row != nullptr) o.ent_row[r] = on ? lab.ent : 0.f;
          o.lse[r] = mt * a.inv_t + ls;
          if (o.lse_rest != nullptr) o.lse_rest[r] = mo > kNegInf ? mo * a.inv_t + lo : kNegInf;
        }
      }
      if (lane == 0) {
        // the greedy token is written by the warp that holds the first of the largest logits outside
        // the list, or by the first warp when the list holds all of them
        sums.top = mo == top ? top : __builtin_nanf("");
        sums.writer = mo == top && top > kNegInf ? first : 0;
        if (!(top > kNegInf)) c = 0.f;
        sums.c = c;
        sums.b = -ls * kLog2e;
        const float olog = ref_residual(mo, k) + lo * kLog2e;   // factors that the fma form carries
        const bool any = mo > kNegInf;
        sums.out_b = any ? ref_offset(mo, k) : 0.f;
        sums.out_c = any ? c * (So * expf(gap) / S - lab.p0) * ex2(-olog) : 0.f;
        sums.ref = mt;
      }
    } else if (lane == 0) {
      const float lse = o.lse[r], lse_rest = rest != nullptr ? o.lse_rest[r] : kNegInf;
      if (!(lse > kNegInf)) c = 0.f;
      sums.c = c;
      sums.ref = 0.f;
      sums.b = lse > kNegInf ? -lse * kLog2e : 0.f;
      if (rest == nullptr) {
        sums.out_b = sums.b;
        sums.out_c = c;
      } else {
        const bool any = lse_rest > kNegInf;
        sums.out_b = any ? -lse_rest * kLog2e : 0.f;
        sums.out_c = any ? c * (expf(lse_rest - lse) - lab.p0) : 0.f;
      }
    }
  }
  if ((kMode & kFwd) && cluster > 1) cluster_arrive();   // no other block's memory is read any more
  __syncthreads();
  if constexpr ((kMode & kFwd) != 0) {
    if (o.argmax != nullptr && rank * n_warps + warp == sums.writer) {
      const float top = sums.top;
      int v = 0x7fffffff;
      float best = top;   // NaN: outside the list there is none
      if (!(top == top)) {
        best = kNegInf;
        for (int i = lane; i < a.K; i += 32)
          if (lab.idx[i] >= 0) best = fmaxf(best, lab.z[i]);
        best = warp_reduce(best, MaxOp());
      } else {
#pragma unroll
        for (int i = 0; i < kPacks; ++i)
#pragma unroll
          for (int e = 0; e < kPerPack<E>; ++e)
            if (pack_elem<E>(raw[i], e) == top) v = min(v, at.elem(i) + e);
      }
      for (int i = lane; i < a.K; i += 32)
        if (lab.idx[i] >= 0 && lab.z[i] == best) v = min(v, lab.idx[i]);
      v = warp_reduce(v, MinOp());
      if (lane == 0) o.argmax[r] = best > kNegInf ? v : -1;
    }
  }
  if constexpr ((kMode & kGrad) != 0) {
    const float c = sums.c, out_b = sums.out_b, out_c = sums.out_c;
    if (c == 0.f) {
#pragma unroll
      for (int i = 0; i < kPacks; ++i) raw[i] = neg_inf_pack<E>();
    }
    const bool aligned = int(r * a.ldg % kPerPack<E>) == at.off;
    if (aligned && at.whole(a.V)) {
      uint4* p = reinterpret_cast<uint4*>(g + at.elem(0));
#pragma unroll
      for (int i = 0; i < kPacks; ++i) {
        const uint4 x = grad_pack<E>(raw[i], k, out_b, out_c);
        const uint32_t skip = listed_bytes[32 * i];
        if (skip == 0)
          __stcs(p + 32 * i, x);
        else
          store_elems(g, at.elem(i), a.V, skip, x);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kPacks; ++i) {
        const int v = at.elem(i);
        const uint4 x = grad_pack<E>(raw[i], k, out_b, out_c);
        const uint32_t skip = listed_bytes[32 * i];
        if (aligned && skip == 0 && v >= 0 && v + kPerPack<E> <= a.V)
          __stcs(reinterpret_cast<uint4*>(g + v), x);
        else
          store_elems(g, v, a.V, skip, x);
      }
    }
    // the listed tokens of this block's range
    for (int i = tid; i < a.K; i += blockDim.x) {
      const int v = lab.idx[i], pack = (v + at.off) / kPerPack<E> - at.base;
      if (v >= 0 && pack >= 0 && pack < n_packs)
        g[v] = E(c != 0.f ? c * (ex2(fmaf(lab.z[i] - sums.ref, k, sums.b)) - lab.p[i]) : 0.f);
    }
  }
  if ((kMode & kFwd) && cluster > 1) cluster_wait();   // until no block reads this one's records
}

// weight_sum = sum of the weights, one block, fixed order.
__global__ void __launch_bounds__(1024)
    weight_sum_kernel(const float* weight, long long N, float* weight_sum) {
  __shared__ double buf[32];
  pdl_wait_and_release();
  double s = 0.0;
  if (weight != nullptr)
    for (long long r = threadIdx.x; r < N; r += 1024) s += double(weight[r]);
  s = block_reduce(s, AddOp(), buf);
  if (threadIdx.x == 0) *weight_sum = weight != nullptr ? float(s) : float(N);
}

// L = lambda sum w l / sum w, one block, fixed order.
__global__ void __launch_bounds__(1024)
    distill_loss_kernel(const float* weight, const float* loss_row, const float* weight_sum,
                        long long N, float lambda, float* loss_total, float* wl_sum) {
  __shared__ double buf[32];
  pdl_wait_and_release();
  double s = 0.0;
  for (long long r = threadIdx.x; r < N; r += 1024)
    s += double(loss_row[r]) * (weight != nullptr ? double(weight[r]) : 1.0);
  s = block_reduce(s, AddOp(), buf);
  if (threadIdx.x == 0) {
    const double ws = *weight_sum;
    *loss_total = ws > 0.0 ? float(double(lambda) * s / ws) : 0.f;
    if (wl_sum != nullptr) *wl_sum = float(s);
  }
}

template <typename E, int kPacks>
cudaError_t launch_rows(const RowShape& shape, const DistillArgs& a, bool fwd, bool grad,
                        const void* Z, const float* top_val, const int32_t* top_idx,
                        const float* rest, const float* weight, const float* weight_sum,
                        const DistillRows& o, void* G, cudaStream_t s) {
  auto kern = fwd ? (grad ? distill_row_kernel<E, kPacks, kFwd | kGrad>
                          : distill_row_kernel<E, kPacks, kFwd>)
                  : distill_row_kernel<E, kPacks, kGrad>;
  return launch_row_clusters(shape, a.N, kern, s, static_cast<const E*>(Z), top_val, top_idx, rest,
                             weight, weight_sum, a, o, static_cast<E*>(G), shape.cluster);
}

}  // namespace

cudaError_t launch_distill(const DistillArgs& a, bool fwd, bool grad, const void* Z,
                           const float* top_val, const int32_t* top_idx, const float* rest,
                           const float* weight, const float* norm, const DistillRows& o,
                           const DistillSums& t, void* G, int sms, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  if (fwd) {
    e = launch_pdl(weight_sum_kernel, dim3(1), dim3(1024), 0, s, weight, a.N, t.weight_sum);
    if (e != cudaSuccess) return e;
    if (norm == nullptr) norm = t.weight_sum;
  }
  if (a.N > 0) {
    const RowShape shape = row_shape(a.N, a.V, a.dtype == 0 ? 2 : 4, sms);
    const auto run = [&](auto packs) {
      constexpr int kP = decltype(packs)::value;
      return a.dtype == 0 ? launch_rows<__nv_bfloat16, kP>(shape, a, fwd, grad, Z, top_val, top_idx,
                                                           rest, weight, norm, o, G, s)
                          : launch_rows<float, kP>(shape, a, fwd, grad, Z, top_val, top_idx, rest,
                                                   weight, norm, o, G, s);
    };
    e = with_packs(shape.packs, run);
    if (e != cudaSuccess) return e;
  }
  if (fwd)
    e = launch_pdl(distill_loss_kernel, dim3(1), dim3(1024), 0, s, weight, o.loss_row,
                   t.weight_sum, a.N, a.lambda, t.loss_total, t.wl_sum);
  return e;
}

}  // namespace alr
