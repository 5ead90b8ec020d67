// Attention of query rows over the paged key-value cache.
#include <algorithm>

#include "kernels.h"
#include "launch.h"
#include "row_reduce.cuh"

namespace alr {
namespace {

// Sequence and length of a row in one of its two parts (its own tokens, its prefix); anything that
// cannot be read counts as no tokens.
struct KvPart {
  const int32_t* seq;   // nullptr: row / per
  const int32_t* len;
  int per;
};

ALR_DEV int part_seq(const KvPart& p, long long row) {
  return p.seq != nullptr ? p.seq[row] : int(row / p.per);
}

ALR_DEV int part_len(const KvAttention& a, const KvPart& p, long long row, int seq) {
  if (seq < 0 || seq >= a.n_seq) return 0;
  return int(min((long long)max(p.len[row], 0), (long long)a.cols * a.c.page));
}

// ------------------------------------------------------------------ row by row ---
// A warp takes one row and head, token by token: lane i holds elements i, i + 32, ... of q and of the
// sum.  (m, l, o): running maximum, sum and weighted values of the scores, in units of log2.
constexpr int kLaneDims = kKvMaxDim / 32;

template <typename E>
ALR_DEV void walk_tokens(const KvAttention& a, int seq, int len, int head,
                         const float (&q)[kLaneDims], float& m, float& l, float (&o)[kLaneDims]) {
  const int lane = threadIdx.x & 31;
  const E* K = static_cast<const E*>(a.c.K) + head * a.c.sh;
  const E* V = static_cast<const E*>(a.c.V) + head * a.c.sh;
  for (int t = 0; t < len; ++t) {
    const int j = t / a.c.page, pg = a.table[(long long)seq * a.cols + j];
    if (pg < 0 || pg >= a.c.n_pages) continue;
    const long long at = pg * a.c.sp + (t - j * a.c.page) * a.c.st;
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < kLaneDims; ++i)
      if (i * 32 + lane < a.c.dim) x = fmaf(q[i], to_float(K[at + i * 32 + lane]), x);
    x = warp_reduce(x, AddOp());
    if (x == kNegInf) continue;
    const float up = fmaxf(m, x), c = ex2(m - up), e = ex2(x - up);
    m = up;
    l = fmaf(l, c, e);
#pragma unroll
    for (int i = 0; i < kLaneDims; ++i)
      if (i * 32 + lane < a.c.dim) o[i] = fmaf(e, to_float(V[at + i * 32 + lane]), o[i] * c);
  }
}

template <typename E>
__global__ void __launch_bounds__(256)
    kv_rows_kernel(const KvAttention a, const KvPart own, const KvPart prefix) {
  pdl_wait_and_release();
  const long long w = (long long)blockIdx.x * 8 + threadIdx.x / 32;
  const long long r = w / a.H;
  if (r >= a.N) return;
  const int h = int(w - r * a.H), lane = threadIdx.x & 31, head = h / (a.H / a.c.heads);
  float q[kLaneDims], o[kLaneDims] = {}, m = kNegInf, l = 0.f;
#pragma unroll
  for (int i = 0; i < kLaneDims; ++i)
    q[i] = i * 32 + lane < a.c.dim
               ? to_float(static_cast<const E*>(a.Q)[r * a.ldq + h * a.c.dim + i * 32 + lane]) *
                     (a.scale * kLog2e)
               : 0.f;
  if (prefix.len != nullptr) {
    const int s = part_seq(prefix, r);
    walk_tokens<E>(a, s, part_len(a, prefix, r, s), head, q, m, l, o);
  }
  const int s = part_seq(own, r);
  walk_tokens<E>(a, s, part_len(a, own, r, s), head, q, m, l, o);
#pragma unroll
  for (int i = 0; i < kLaneDims; ++i)
    if (i * 32 + lane < a.c.dim)
      static_cast<E*>(a.out)[r * a.ldo + h * a.c.dim + i * 32 + lane] = E(l == 0.f ? 0.f : o[i] / l);
  if (lane == 0 && a.lse != nullptr) a.lse[r * a.H + h] = l == 0.f ? kNegInf : m * kLn2 + logf(l);
}

}  // namespace

size_t kv_attention_workspace(long long N, int H, int dim, bool prefix) { return 16; }

cudaError_t launch_kv_attention(const KvAttention& a, int sms, int* status, cudaStream_t s) {
  const KvPart own = {a.seq, a.len, a.rows_per_seq};
  const KvPart prefix = {a.prefix_seq, a.prefix_len, a.rows_per_prefix};
  const long long warps = a.N * a.H;
  const dim3 grid(unsigned((warps + 7) / 8));
  if (a.c.dtype == 0)
    return launch_pdl(kv_rows_kernel<__nv_bfloat16>, grid, dim3(256), 0, s, a, own, prefix);
  return launch_pdl(kv_rows_kernel<float>, grid, dim3(256), 0, s, a, own, prefix);
}

}  // namespace alr
