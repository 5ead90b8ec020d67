// Reductions over the threads of a block, and the order of logits, for the kernels that walk rows of
// logits (distill_kernels.cu, sample_kernels.cu).
#pragma once

#include <cuda_bf16.h>

#include "tc_common.cuh"

namespace alr {

constexpr float kNegInf = -__builtin_huge_valf();

ALR_DEV float to_float(float x) { return x; }
ALR_DEV float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

struct MaxOp {
  template <typename T>
  ALR_DEV T operator()(T a, T b) const { return a > b ? a : b; }
};
struct AddOp {
  template <typename T>
  ALR_DEV T operator()(T a, T b) const { return a + b; }
};

template <typename T, typename Op>
ALR_DEV T warp_reduce(T v, Op op) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, off));
  return v;
}

// Sum of the lanes up to and with this one.
template <typename T>
ALR_DEV T warp_scan(T v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const T t = __shfl_up_sync(0xffffffffu, v, off);
    if (lane >= off) v += t;
  }
  return v;
}

// Largest float of the warp, in one instruction (NaN is not passed).
ALR_DEV float warp_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
ALR_DEV int warp_min(int v) { return __reduce_min_sync(0xffffffffu, v); }

// op over the values of all threads of the block (a multiple of 32, at most 1024), in a fixed
// order; every thread gets the result.  `buf`: 32 entries of shared memory, free again on return.
template <typename T, typename Op>
ALR_DEV T block_reduce(T v, Op op, T* buf) {
  v = warp_reduce(v, op);
  const int lane = threadIdx.x & 31, n_warps = blockDim.x / 32;
  if (lane == 0) buf[threadIdx.x / 32] = v;
  __syncthreads();
  T r = buf[lane < n_warps ? lane : 0];
  // lanes past the warps repeat warp 0's value: harmless to a minimum or maximum, left out of a sum
  if constexpr (sizeof(Op) == sizeof(AddOp) && __is_same(Op, AddOp))
    if (lane >= n_warps) r = T(0);
  r = warp_reduce(r, op);
  __syncthreads();
  return r;
}

// Monotone map of a finite or infinite float to an unsigned key: a < b as floats means a smaller key;
// -0 and +0 get the same key.  NaN is never passed.
ALR_DEV uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(__fadd_rn(x, 0.f));
  return b ^ (int32_t(b) < 0 ? 0xffffffffu : 0x80000000u);
}
ALR_DEV float key_value(uint32_t k) {
  return __uint_as_float(k ^ (int32_t(k) < 0 ? 0x80000000u : 0xffffffffu));
}

}  // namespace alr
