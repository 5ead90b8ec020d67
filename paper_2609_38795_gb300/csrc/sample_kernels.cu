// A teacher's top logits, and the next token of a rollout drawn from given random numbers.
//
// Both pick from a row by the order (value descending, token id ascending).  A logit that is -inf or
// NaN is no candidate.  Selection is a radix select over the 8-bit digits of an order-preserving
// 32-bit key; equal values at the threshold go to the lowest ids.
#include "kernels.h"
#include "launch.h"
#include "row_reduce.cuh"

namespace alr {
namespace {

constexpr int kRowThreads = 512;

// What a row keeps: keys above `key`, and of the tokens with that key those up to id `last`.
struct Cut {
  uint32_t key;
  int last;
  ALR_DEV bool keeps(uint32_t k, int v) const { return k > key || (k == key && v <= last); }
};

struct SelectShared {
  unsigned long long hist[256];
  unsigned long long scan[256];
  uint32_t prefix;
  unsigned long long above;
  int count[32];
  int found;
  float buf[32];
  unsigned long long lbuf[32];
  int ibuf[32];
};

// The token with the n-th lowest id (n >= 1) among those with `key` that `cut` keeps.
template <typename E>
ALR_DEV int nth_equal(const E* z, int V, const Cut& cut, uint32_t key, long long n,
                      SelectShared& sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, n_warps = blockDim.x / 32;
  if (threadIdx.x == 0) sh.found = V - 1;
  long long before = 0;
  __syncthreads();
  for (int base = 0; base < V; base += blockDim.x) {
    const int v = base + threadIdx.x;
    bool is = false;
    if (v < V) {
      const float x = to_float(z[v]);
      is = x > kNegInf && order_key(x) == key && cut.keeps(key, v);
    }
    const unsigned ball = __ballot_sync(0xffffffffu, is);
    if (lane == 0) sh.count[warp] = __popc(ball);
    __syncthreads();
    long long mine = before, all = 0;
    for (int w = 0; w < n_warps; ++w) {
      if (w < warp) mine += sh.count[w];
      all += sh.count[w];
    }
    mine += __popc(ball & ((2u << lane) - 1u));
    if (is && mine == n) sh.found = v;
    before += all;
    __syncthreads();
    if (before >= n) break;
  }
  return sh.found;
}

// The key at which the summed weights of the kept tokens, from the largest key down, first reach
// more than... `need(above)` says whether a sum `above` of all larger keys still lacks something.
// weight(x): whole weight of a token.  Returns the key; `above` gets the sum over larger keys.
template <typename E, typename W, typename Need>
ALR_DEV uint32_t select_key(const E* z, int V, const Cut& cut, W weight, Need need,
                            unsigned long long& above_out, SelectShared& sh) {
  uint32_t prefix = 0;
  unsigned long long above = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += blockDim.x) sh.hist[i] = 0;
    __syncthreads();
    for (int v = threadIdx.x; v < V; v += blockDim.x) {
      const float x = to_float(z[v]);
      if (!(x > kNegInf)) continue;
      const uint32_t k = order_key(x);
      if (!cut.keeps(k, v)) continue;
      if (shift < 24 && (k >> (shift + 8)) != (prefix >> (shift + 8))) continue;
      atomicAdd(&sh.hist[(k >> shift) & 255], weight(x));
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      int d = 255;
      for (; d > 0; --d) {   // the digit whose bin the need ends in
        if (sh.hist[d] != 0 && !need(above + sh.hist[d])) break;
        above += sh.hist[d];
      }
      sh.prefix = prefix | (uint32_t(d) << shift);
      sh.above = above;
    }
    __syncthreads();
    prefix = sh.prefix;
    above = sh.above;
    __syncthreads();
  }
  above_out = above;
  return prefix;
}

// The cut that keeps the k first tokens (k >= 1) of the row.
template <typename E>
ALR_DEV Cut cut_top_k(const E* z, int V, long long k, SelectShared& sh) {
  const Cut all{0u, 0x7fffffff};
  unsigned long long above;
  const uint32_t key = select_key(
      z, V, all, [](float) { return 1ull; },
      [k](unsigned long long got) { return got < (unsigned long long)k; }, above, sh);
  return {key, nth_equal(z, V, all, key, k - (long long)above, sh)};
}

// ---------------------------------------------------------------- top logits ---
template <typename E>
__global__ void __launch_bounds__(kRowThreads)
    top_logits_kernel(const E* Z, long long ldz, int V, int K, float inv_t, float* top_val,
                      int32_t* top_idx, float* lse, float* lse_rest) {
  __shared__ SelectShared sh;
  __shared__ uint32_t key[kTopMost];
  __shared__ int id[kTopMost];
  __shared__ int n_got;
  pdl_wait_and_release();
  const long long r = blockIdx.x;
  const E* z = Z + r * ldz;
  float m = kNegInf;
  int finite = 0;
  for (int v = threadIdx.x; v < V; v += blockDim.x) {
    const float x = to_float(z[v]);
    if (x > kNegInf) {
      m = fmaxf(m, x);
      ++finite;
    }
  }
  m = block_reduce(m, MaxOp(), sh.buf);
  finite = block_reduce(finite, AddOp(), sh.ibuf);
  const int n = min(K, finite);
  Cut cut{0xffffffffu, -1};
  if (n > 0) cut = cut_top_k(z, V, n, sh);
  if (threadIdx.x == 0) n_got = 0;
  __syncthreads();
  const float c = inv_t * kLog2e;
  // the tokens not listed are summed from their own maximum: what they hold next to the listed ones
  // may be below the range of the largest one's exponential
  float mo = kNegInf;
  for (int v = threadIdx.x; v < V; v += blockDim.x) {
    const float x = to_float(z[v]);
    if (!(x > kNegInf)) continue;
    const uint32_t k = order_key(x);
    if (cut.keeps(k, v)) {
      const int at = atomicAdd(&n_got, 1);
      if (at < kTopMost) {
        key[at] = k;
        id[at] = v;
      }
    } else {
      mo = fmaxf(mo, x);
    }
  }
  mo = block_reduce(mo, MaxOp(), sh.buf);
  float So = 0.f, S = 0.f;
  for (int v = threadIdx.x; v < V; v += blockDim.x) {
    const float x = to_float(z[v]);
    if (x > kNegInf && !cut.keeps(order_key(x), v)) So += ex2((x - mo) * c);
  }
  So = block_reduce(So, AddOp(), sh.buf);
  for (int i = threadIdx.x; i < n; i += blockDim.x) S += ex2((key_value(key[i]) - m) * c);
  S = block_reduce(S, AddOp(), sh.buf);
  if (mo > kNegInf) S += So * ex2((mo - m) * c);
  // an entry's place is the number of entries before it in the order
  for (int i = threadIdx.x; i < K; i += blockDim.x) {
    if (i < n) {
      int place = 0;
      for (int j = 0; j < n; ++j)
        place += key[j] > key[i] || (key[j] == key[i] && id[j] < id[i]);
      top_val[r * K + place] = key_value(key[i]);
      top_idx[r * K + place] = id[i];
    } else {
      top_val[r * K + i] = kNegInf;
      top_idx[r * K + i] = -1;
    }
  }
  if (threadIdx.x == 0) {
    if (lse != nullptr) lse[r] = n > 0 ? m * inv_t + logf(S) : kNegInf;
    if (lse_rest != nullptr) lse_rest[r] = mo > kNegInf ? mo * inv_t + logf(So) : kNegInf;
  }
}

// ------------------------------------------------------------------ sampling ---
// A token's weight is the whole number floor(2^31 exp2((z - max) c)), c = log2 e / temperature, every
// step rounded to fp32 on its own: sums of weights are exact, so neither the order of summation nor
// the split of a row over threads can change a draw.
struct Weight {
  float m, c;
  ALR_DEV float real(float x) const { return x == m ? 1.f : exp2f(__fmul_rn(__fsub_rn(x, m), c)); }
  ALR_DEV unsigned long long operator()(float x) const {
    return (unsigned long long)(real(x) * 2147483648.f);
  }
};

template <typename E>
__global__ void __launch_bounds__(kRowThreads)
    sample_kernel(const E* Z, long long ldz, int V, SampleArgs a, int32_t* token, float* prob,
                  int32_t* n_kept) {
  __shared__ SelectShared sh;
  pdl_wait_and_release();
  const long long r = blockIdx.x;
  const E* z = Z + r * ldz;
  float m = kNegInf;
  int at = 0x7fffffff;
  for (int v = threadIdx.x; v < V; v += blockDim.x) {
    const float x = to_float(z[v]);
    if (x > m) {
      m = x;
      at = v;
    }
  }
  const float top = block_reduce(m, MaxOp(), sh.buf);
  const int first = block_reduce(m == top ? at : 0x7fffffff, MinOp(), sh.ibuf);
  const float T = a.temperature != nullptr ? a.temperature[r] : 1.f;
  if (!(top > kNegInf) || !(T > 0.f)) {
    if (threadIdx.x == 0) {
      const bool some = top > kNegInf;
      token[r] = some ? first : -1;
      if (prob != nullptr) prob[r] = some ? 1.f : 0.f;
      if (n_kept != nullptr) n_kept[r] = some ? 1 : 0;
    }
    return;
  }
  const Weight weight{top, __fdiv_rn(kLog2e, T)};
  Cut cut{0u, 0x7fffffff};
  const int k = a.top_k != nullptr ? a.top_k[r] : 0;
  if (k > 0 && k < V) {
    int finite = 0;
    for (int v = threadIdx.x; v < V; v += blockDim.x) finite += to_float(z[v]) > kNegInf;
    finite = block_reduce(finite, AddOp(), sh.ibuf);
    if (k < finite) cut = cut_top_k(z, V, k, sh);
  }
  const float min_p = a.min_p != nullptr ? fminf(a.min_p[r], 1.f) : 0.f;
  auto total = [&](int& count, float least) {
    unsigned long long s = 0;
    int n = 0;
    for (int v = threadIdx.x; v < V; v += blockDim.x) {
      const float x = to_float(z[v]);
      if (!(x > kNegInf) || !cut.keeps(order_key(x), v)) continue;
      const unsigned long long w = weight(x);
      if (w == 0 || (x != top && weight.real(x) < least)) continue;
      s += w;
      ++n;
    }
    count = block_reduce(n, AddOp(), sh.ibuf);
    return block_reduce(s, AddOp(), sh.lbuf);
  };
  const float top_p = a.top_p != nullptr ? a.top_p[r] : 1.f;
  int n = 0;
  if (top_p < 1.f) {
    const double lim = double(top_p) * double(total(n, 0.f));
    unsigned long long above;
    const uint32_t key = select_key(
        z, V, cut, weight, [lim](unsigned long long got) { return double(got) < lim; }, above, sh);
    // tokens with this key while the sum before them is below the limit, one at least
    const unsigned long long w = weight(key_value(key));
    long long more = 1;
    if (w > 0) {
      more = (long long)((lim - double(above)) / double(w));
      more = more < 1 ? 1 : more;
      while (more > 1 && !(double(above + (more - 1) * w) < lim)) --more;
      while (double(above + more * w) < lim) ++more;
    }
    cut = {key, nth_equal(z, V, cut, key, more, sh)};
  }
  const unsigned long long S = total(n, min_p);
  // floor(u S / 2^32): the first token, in the order of ids, whose running sum exceeds it
  const unsigned long long u = a.u[r];
  const unsigned long long target = __umul64hi(u << 32, S);
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, n_warps = blockDim.x / 32;
  unsigned long long before = 0;
  for (int base = 0; base < V; base += blockDim.x) {
    const int v = base + threadIdx.x;
    unsigned long long w = 0;
    if (v < V) {
      const float x = to_float(z[v]);
      if (x > kNegInf && cut.keeps(order_key(x), v)) {
        w = weight(x);
        if (x != top && weight.real(x) < min_p) w = 0;
      }
    }
    unsigned long long incl = w;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const unsigned long long t = __shfl_up_sync(0xffffffffu, incl, off);
      if (lane >= off) incl += t;
    }
    if (lane == 31) sh.lbuf[warp] = incl;
    __syncthreads();
    unsigned long long mine = before, all = 0;
    for (int i = 0; i < n_warps; ++i) {
      if (i < warp) mine += sh.lbuf[i];
      all += sh.lbuf[i];
    }
    if (w > 0 && mine + incl - w <= target && mine + incl > target) {
      token[r] = v;
      if (prob != nullptr) prob[r] = float(double(w) / double(S));
    }
    before += all;
    __syncthreads();
    if (before > target) break;
  }
  if (threadIdx.x == 0 && n_kept != nullptr) n_kept[r] = n;
}

}  // namespace

cudaError_t launch_top_logits(int dtype, const void* Z, long long N, int V, long long ldz, int K,
                              float inv_t, float* top_val, int32_t* top_idx, float* lse,
                              float* lse_rest, cudaStream_t s) {
  if (dtype == 0)
    return launch_pdl(top_logits_kernel<__nv_bfloat16>, dim3(unsigned(N)), dim3(kRowThreads), 0, s,
                      static_cast<const __nv_bfloat16*>(Z), ldz, V, K, inv_t, top_val, top_idx, lse,
                      lse_rest);
  return launch_pdl(top_logits_kernel<float>, dim3(unsigned(N)), dim3(kRowThreads), 0, s,
                    static_cast<const float*>(Z), ldz, V, K, inv_t, top_val, top_idx, lse,
                    lse_rest);
}

cudaError_t launch_sample(int dtype, const void* Z, long long N, int V, long long ldz,
                          const SampleArgs& a, int32_t* token, float* prob, int32_t* n_kept,
                          cudaStream_t s) {
  if (dtype == 0)
    return launch_pdl(sample_kernel<__nv_bfloat16>, dim3(unsigned(N)), dim3(kRowThreads), 0, s,
                      static_cast<const __nv_bfloat16*>(Z), ldz, V, a, token, prob, n_kept);
  return launch_pdl(sample_kernel<float>, dim3(unsigned(N)), dim3(kRowThreads), 0, s,
                    static_cast<const float*>(Z), ldz, V, a, token, prob, n_kept);
}

}  // namespace alr
