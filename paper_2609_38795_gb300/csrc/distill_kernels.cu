// Distillation from a teacher's top logits: the loss of student logits in hand, and its gradient.
//
// Label of a row: softmax over the teacher's listed logits t_i / T and, when given, the log-sum-exp
// of the tokens that are not listed (one bin for all of them).  With s = z / T, m = max s,
// S = sum exp(s - m), R = log-sum-exp of s over the tokens not listed:
//   l = log S + sum_i p_i (m - s_i) + p_0 (m - R)        (no large numbers cancel)
//   dl / dz_v = (q_v - p_v) / T for a listed v, else q_v (1 - p_0 / q_0) / T,   q = exp(s) / sum.
// A bitmap of the listed tokens in shared memory keeps them out of R's sum, which is taken from the
// largest logit outside the list: exact however small the mass there is (taking the listed terms
// off the whole sum would leave rounding errors of the size of the list's own).  Differences of
// logits are taken before the division by T: they are exact for neighbours.
#include "kernels.h"
#include "launch.h"
#include "row_reduce.cuh"

namespace alr {
namespace {

constexpr int kRowThreads = 512;

struct Label {
  float p;     // this thread's probability (threads >= K: 0)
  float p0;    // the tail bin's
  float ent;   // entropy of the label
  bool has;    // some probability is positive
  int idx;     // this thread's token, -1 for none
};

// The row's label; thread i holds entry i.
ALR_DEV Label row_label(const float* top_val, const int32_t* top_idx, const float* rest,
                        const DistillArgs& a, long long r, float* buf) {
  Label l{};
  l.idx = -1;
  float x = kNegInf;
  if (int(threadIdx.x) < a.K) {
    const int v = top_idx[r * a.K + threadIdx.x];
    if (v >= 0 && v < a.V) {
      l.idx = v;
      x = top_val[r * a.K + threadIdx.x];
    }
  }
  const float x0 = rest != nullptr ? rest[r] : kNegInf;
  const float tm = block_reduce(x, MaxOp(), buf), m = fmaxf(tm * a.inv_t, x0);
  l.has = m > kNegInf;
  if (!l.has) return l;
  const float step = tm > kNegInf ? tm * a.inv_t - m : 0.f;     // 0 unless the bin leads
  x = x > kNegInf ? (x - tm) * a.inv_t + step : kNegInf;
  const float d0 = x0 - m;
  const float e = x > kNegInf ? expf(x) : 0.f, e0 = d0 > kNegInf ? expf(d0) : 0.f;
  const float sum = block_reduce(e, AddOp(), buf) + e0;
  const float ls = logf(sum);
  l.p = e / sum;
  l.p0 = e0 / sum;
  // H = sum p (log sum - x)
  const float h = l.p > 0.f ? l.p * (ls - x) : 0.f;
  l.ent = block_reduce(h, AddOp(), buf) + (l.p0 > 0.f ? l.p0 * (ls - d0) : 0.f);
  return l;
}

// One block per row.  kFwd: the row's loss, entropy, log-sum-exps and greedy token; kGrad: the
// gradient of its logits, from this row's sums (both) or from lse, lse_rest of an earlier forward.
template <typename E, bool kFwd, bool kGrad>
__global__ void __launch_bounds__(kRowThreads)
    distill_row_kernel(const E* Z, const float* top_val, const int32_t* top_idx, const float* rest,
                       const float* weight, const float* weight_sum, DistillArgs a,
                       DistillRows o, E* G) {
  extern __shared__ uint32_t in_list[];
  __shared__ float buf[32];
  __shared__ int ibuf[32];
  pdl_wait_and_release();
  const long long r = blockIdx.x;
  const E* z = Z + r * a.ldz;
  E* g = G + r * a.ldg;
  const float w = weight != nullptr ? weight[r] : 1.f;
  if (w == 0.f) {   // not read
    if (kFwd && threadIdx.x == 0) {
      o.loss_row[r] = 0.f;
      if (o.ent_row != nullptr) o.ent_row[r] = 0.f;
      o.lse[r] = 0.f;
      if (o.lse_rest != nullptr) o.lse_rest[r] = 0.f;
      if (o.argmax != nullptr) o.argmax[r] = -1;
    }
    if constexpr (kGrad)
      for (int v = threadIdx.x; v < a.V; v += kRowThreads) g[v] = E(0.f);
    return;
  }
  for (int i = threadIdx.x; i < (a.V + 31) / 32; i += kRowThreads) in_list[i] = 0;
  const Label l = row_label(top_val, top_idx, rest, a, r, buf);
  __syncthreads();
  if (l.idx >= 0) atomicOr(&in_list[l.idx >> 5], 1u << (l.idx & 31));
  const float z_i = l.idx >= 0 ? to_float(z[l.idx]) : kNegInf;
  __syncthreads();
  float lse, lse_rest;
  if constexpr (kFwd) {
    float m = kNegInf, mo = kNegInf;
    int at = 0x7fffffff;
    for (int v = threadIdx.x; v < a.V; v += kRowThreads) {
      const float x = to_float(z[v]);
      if (x > m) {
        m = x;
        at = v;
      }
      if (!(in_list[v >> 5] >> (v & 31) & 1)) mo = fmaxf(mo, x);
    }
    const float top = block_reduce(m, MaxOp(), buf);
    const int first = block_reduce(m == top ? at : 0x7fffffff, MinOp(), ibuf);
    mo = block_reduce(mo, MaxOp(), buf);
    const float mt = top > kNegInf ? top : 0.f, c = a.inv_t * kLog2e;
    float So = 0.f;
    if (mo > kNegInf)
      for (int v = threadIdx.x; v < a.V; v += kRowThreads)
        if (!(in_list[v >> 5] >> (v & 31) & 1)) So += ex2((to_float(z[v]) - mo) * c);
    So = block_reduce(So, AddOp(), buf);
    const float step = mo > kNegInf ? (mo - mt) * a.inv_t : kNegInf;
    float S = block_reduce(l.idx >= 0 ? ex2((z_i - mt) * c) : 0.f, AddOp(), buf);
    if (mo > kNegInf) S += So * expf(step);
    const float ls = logf(S), lo = logf(So) + step;
    lse = mt * a.inv_t + ls;
    lse_rest = mo > kNegInf ? mo * a.inv_t + logf(So) : kNegInf;
    const float li = l.p > 0.f ? l.p * (ls + (mt - z_i) * a.inv_t) : 0.f;
    const float loss = block_reduce(li, AddOp(), buf) + (l.p0 > 0.f ? l.p0 * (ls - lo) : 0.f);
    if (threadIdx.x == 0) {
      const bool on = l.has && top > kNegInf;
      o.loss_row[r] = on ? loss : 0.f;
      if (o.ent_row != nullptr) o.ent_row[r] = on ? l.ent : 0.f;
      o.lse[r] = lse;
      if (o.lse_rest != nullptr) o.lse_rest[r] = lse_rest;
      if (o.argmax != nullptr) o.argmax[r] = top > kNegInf ? first : -1;
    }
  } else {
    lse = o.lse[r];
    lse_rest = rest != nullptr ? o.lse_rest[r] : kNegInf;
  }
  if constexpr (kGrad) {
    const float ws = *weight_sum;
    const float c = l.has && lse > kNegInf && ws > 0.f ? a.lambda * w / ws * a.inv_t : 0.f;
    const float k = a.inv_t * kLog2e;
    // outside the list q_v (1 - p_0 / q_0); q_0 = 0 leaves no token there
    const float beta = l.p0 > 0.f && lse_rest > kNegInf ? 1.f - l.p0 * expf(lse - lse_rest) : 1.f;
    const float b = lse > kNegInf ? -lse * kLog2e : 0.f;
    for (int v = threadIdx.x; v < a.V; v += kRowThreads) {
      if (in_list[v >> 5] >> (v & 31) & 1) continue;
      g[v] = E(c != 0.f ? c * beta * ex2(fmaf(to_float(z[v]), k, b)) : 0.f);
    }
    if (l.idx >= 0) g[l.idx] = E(c != 0.f ? c * (ex2(fmaf(z_i, k, b)) - l.p) : 0.f);
  }
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

template <typename E>
cudaError_t launch_rows(const DistillArgs& a, bool fwd, bool grad, const void* Z,
                        const float* top_val, const int32_t* top_idx, const float* rest,
                        const float* weight, const float* weight_sum, const DistillRows& o, void* G,
                        cudaStream_t s) {
  auto kern = fwd ? (grad ? distill_row_kernel<E, true, true> : distill_row_kernel<E, true, false>)
                  : distill_row_kernel<E, false, true>;
  const size_t smem = size_t((a.V + 31) / 32) * 4;
  return launch_pdl(kern, dim3(unsigned(a.N)), dim3(kRowThreads), smem, s,
                    static_cast<const E*>(Z), top_val, top_idx, rest, weight, weight_sum, a, o,
                    static_cast<E*>(G));
}

}  // namespace

cudaError_t launch_distill(const DistillArgs& a, bool fwd, bool grad, const void* Z,
                           const float* top_val, const int32_t* top_idx, const float* rest,
                           const float* weight, const float* norm, const DistillRows& o,
                           const DistillSums& t, void* G, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  if (fwd) {
    e = launch_pdl(weight_sum_kernel, dim3(1), dim3(1024), 0, s, weight, a.N, t.weight_sum);
    if (e != cudaSuccess) return e;
    if (norm == nullptr) norm = t.weight_sum;
  }
  if (a.N > 0) {
    e = a.dtype == 0 ? launch_rows<__nv_bfloat16>(a, fwd, grad, Z, top_val, top_idx, rest, weight,
                                                  norm, o, G, s)
                     : launch_rows<float>(a, fwd, grad, Z, top_val, top_idx, rest, weight, norm, o,
                                          G, s);
    if (e != cudaSuccess) return e;
  }
  if (fwd)
    e = launch_pdl(distill_loss_kernel, dim3(1), dim3(1024), 0, s, weight, o.loss_row,
                   t.weight_sum, a.N, a.lambda, t.loss_total, t.wl_sum);
  return e;
}

}  // namespace alr
