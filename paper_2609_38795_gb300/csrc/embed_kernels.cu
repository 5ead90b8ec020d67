// Embedding of tokens, scaled, and the gradient of the table.
#include "kernels.h"
#include "launch.h"
#include "row_reduce.cuh"

namespace alr {
namespace {

constexpr int kEmbedThreads = 256;

// out[i] = scale * E[token_i] (fp32 product, rounded once); a token outside [0, V) gives zeros.
template <typename E>
__global__ void __launch_bounds__(kEmbedThreads)
    embed_kernel(const E* table, int V, int d, const int32_t* tokens, float scale, E* out) {
  pdl_wait_and_release();
  const long long i = blockIdx.x;
  const int v = tokens[i];
  const bool ok = v >= 0 && v < V;
  const E* src = table + (ok ? (long long)v * d : 0);
  for (int c = threadIdx.x; c < d; c += kEmbedThreads)
    out[i * d + c] = ok ? E(to_float(src[c]) * scale) : E(0.f);
}

// One block per token: the first row of each token adds up its rows in order.
template <typename E>
__global__ void __launch_bounds__(kEmbedThreads)
    embed_grad_kernel(const E* dY, int V, int d, const int32_t* tokens, int N, float scale,
                      float* dE) {
  __shared__ int buf[32];
  pdl_wait_and_release();
  const int i = blockIdx.x, v = tokens[i];
  if (v < 0 || v >= V) return;
  int before = 0;
  for (int j = threadIdx.x; j < i; j += kEmbedThreads) before |= tokens[j] == v;
  if (block_reduce(before, MaxOp(), buf) != 0) return;
  for (int c = threadIdx.x; c < d; c += kEmbedThreads) {
    float s = 0.f;
    for (int j = i; j < N; ++j)
      if (tokens[j] == v) s += to_float(dY[(long long)j * d + c]);
    dE[(long long)v * d + c] += scale * s;
  }
}

}  // namespace

cudaError_t launch_embed(int dtype, const void* table, int V, int d, const int32_t* tokens,
                         long long N, float scale, void* out, cudaStream_t s) {
  if (dtype == 0)
    return launch_pdl(embed_kernel<__nv_bfloat16>, dim3(unsigned(N)), dim3(kEmbedThreads), 0, s,
                      static_cast<const __nv_bfloat16*>(table), V, d, tokens, scale,
                      static_cast<__nv_bfloat16*>(out));
  return launch_pdl(embed_kernel<float>, dim3(unsigned(N)), dim3(kEmbedThreads), 0, s,
                    static_cast<const float*>(table), V, d, tokens, scale,
                    static_cast<float*>(out));
}

cudaError_t launch_embed_grad(int dtype, const void* dY, int V, int d, const int32_t* tokens,
                              int N, float scale, bool accumulate, float* dE, void* workspace,
                              cudaStream_t s) {
  (void)workspace;
  if (!accumulate) {
    const cudaError_t e = cudaMemsetAsync(dE, 0, sizeof(float) * size_t(V) * size_t(d), s);
    if (e != cudaSuccess) return e;
  }
  if (N == 0) return cudaSuccess;
  if (dtype == 0)
    return launch_pdl(embed_grad_kernel<__nv_bfloat16>, dim3(unsigned(N)), dim3(kEmbedThreads), 0,
                      s, static_cast<const __nv_bfloat16*>(dY), V, d, tokens, N, scale, dE);
  return launch_pdl(embed_grad_kernel<float>, dim3(unsigned(N)), dim3(kEmbedThreads), 0, s,
                    static_cast<const float*>(dY), V, d, tokens, N, scale, dE);
}

size_t embed_grad_workspace(int, int, int) { return 16; }

}  // namespace alr
