// Attention of query rows over the paged key-value cache, up to 16 queries of a tile at a time.
#include <algorithm>
#include <cfloat>

#include "launch.h"
#include "kv_tiles.cuh"

namespace alr {
namespace {

// ------------------------------------------------------------------------- cores ---
// A core holds the sums of an item's queries for a warp: load_q, see (how many tokens of the run each of
// the lane's queries sees), add (one block from the ring), leave (the sums to shared memory).
//   A token's row in shared memory is `row` bytes, its elements and 16 more where that makes an odd number
// of packs of 16 bytes, so that eight rows' packs at the same place fall in different banks.
constexpr int kNoQuery = INT_MAX;
constexpr float kNoRef = -FLT_MAX;

ALR_DEV void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
ALR_DEV void ldmatrix4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
ALR_DEV void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Transpose of an 8 x 8 matrix of 16-bit elements, two of a row in each lane.
ALR_DEV uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
ALR_DEV uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// A maximum that a running reference may lag behind by (log2): weights up to 2^8 relative to it, and the
// sums are scaled only when it moves, a few times an item.
constexpr float kLag = 8.f;

// bf16 on tensor cores (m16n8k16, fp32 accumulation).  Queries are the 16 rows of a product's result, so
// the weights leave the first product in the registers that the second takes them from.  Lane
// (g, t) = (lane / 4, lane % 4) has queries g and g + 8.
//   16 tokens of 128 elements are 8 KB and 32 product instructions, whatever part of the 16 rows is used
// (64 sequences of 1000 to 3000 tokens, 4 heads of 128, 16 queries each: 262 MB in 101 us cold).
template <int kDim_>
struct ManyCore {
  using E = __nv_bfloat16;
  static constexpr int kBlk = 16;            // tokens of a block
  static constexpr int kDim = kDim_, kMostWarps = 8, kMaxQ = 16;
  static constexpr int kSteps = kDim / 16, kPacks = kDim / 8;
  static constexpr int kScratch = 0;
  int lim[2];
  uint32_t q[kSteps][4];
  float o[kDim / 8][4];
  float m[2], l[2];
  bool two;                                  // more than 8 queries

  // n_q: queries, p.gw a row; of a row's the first `gw` exist.
  ALR_DEV void load_q(const KvPass& p, long long row0, int h0, int n_q, int gw, void*) {
    const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
    two = n_q > 8;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int i = g + 8 * half, r = i / p.gw;
      const bool there = i < n_q && i - r * p.gw < gw;
      const E* src = static_cast<const E*>(p.a.Q) +
                     (there ? (row0 + r) * p.a.ldq + (h0 + i - r * p.gw) * p.a.c.dim : 0);
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int d = k * 16 + e * 8 + 2 * t;
          q[k][half + 2 * e] = there && d < p.a.c.dim ? *reinterpret_cast<const uint32_t*>(src + d) : 0u;
        }
    }
  }
  ALR_DEV void zero() {
    m[0] = m[1] = kNegInf;
    l[0] = l[1] = 0.f;
#pragma unroll
    for (int i = 0; i < kDim / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  }
  // tokens: of the run, by row (lane)
  ALR_DEV void see(const KvPass& p, int tokens, int n_q) {
    const int g = (threadIdx.x & 31) >> 2;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int v = __shfl_sync(~0u, tokens, ((g + 8 * h) / p.gw) & 31);
      lim[h] = g + 8 * h < n_q ? v : kNoQuery;
    }
  }
  // t0: the block's first token; there: tokens whose page exists; plain: all of them seen by all queries.
  ALR_DEV void add(const KvPass& p, char* ring, int row_bytes, int t0, uint32_t there, bool plain, void*) {
    const int lane = threadIdx.x & 31, t = lane & 3;
    const uint32_t k_at = smem_u32(ring), v_at = k_at + kBlk * row_bytes;
    float s[2][4] = {};
    {
      const int row = (lane >> 4) * 8 + (lane & 7), c = lane >> 3 & 1;
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        if (k * 16 >= p.a.c.dim) break;
        uint32_t b[4];
        ldmatrix4(b, k_at + row * row_bytes + 16 * (2 * k + c));
        mma_16816(s[0], q[k], b[0], b[1]);
        mma_16816(s[1], q[k], b[2], b[3]);
      }
    }
    const float c = p.a.scale * kLog2e;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] = __fmul_rn(s[n][e], c);   // never an fma with the reference
    if (!plain) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int tok = n * 8 + 2 * t + (e & 1);
          if (t0 + tok >= lim[e >> 1] || !(there >> tok & 1)) s[n][e] = kNegInf;
        }
    }
    float top[2];
    bool moves = false;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      top[h] = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
      top[h] = fmaxf(top[h], __shfl_xor_sync(~0u, top[h], 1));
      top[h] = fmaxf(top[h], __shfl_xor_sync(~0u, top[h], 2));
      moves |= top[h] > m[h] + kLag;
    }
    if (__any_sync(~0u, moves)) {
      float f[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float up = fmaxf(m[h], top[h]);
        f[h] = m[h] == up ? 1.f : ex2(m[h] - up);
        m[h] = up;
        l[h] *= f[h];
      }
#pragma unroll
      for (int i = 0; i < kDim / 8; ++i) {
        o[i][0] *= f[0], o[i][1] *= f[0];
        o[i][2] *= f[1], o[i][3] *= f[1];
      }
    }
    uint32_t w[4] = {};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h == 1 && !two) break;
      const float ref = m[h] == kNegInf ? 0.f : m[h];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float a = ex2(s[n][2 * h] - ref), b = ex2(s[n][2 * h + 1] - ref);
        l[h] += a + b;
        w[h + 2 * n] = pack_bf16(a, b);     // the product's only operand type: off by 2^-8, l is not
      }
    }
    const int row = (lane >> 3 & 1) * 8 + (lane & 7), c2 = lane >> 4;
#pragma unroll
    for (int i = 0; i < kDim / 16; ++i) {
      if (i * 16 >= p.a.c.dim) break;
      uint32_t b[4];
      ldmatrix4_t(b, v_at + row * row_bytes + 16 * (2 * i + c2));
      mma_16816(o[2 * i], w, b[0], b[1]);
      mma_16816(o[2 * i + 1], w, b[2], b[3]);
    }
  }
  // The sums into shared memory: o as rows of dim + 4, m and l behind n_q of them.
  ALR_DEV void leave(int n_q, int dim, float* to) {
    const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
    float* ml = to + n_q * (dim + 4);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      l[h] += __shfl_xor_sync(~0u, l[h], 1);
      l[h] += __shfl_xor_sync(~0u, l[h], 2);
      const int i = g + 8 * h;
      if (i < n_q) {
        if (t == 0) ml[2 * i] = m[h], ml[2 * i + 1] = l[h];
#pragma unroll
        for (int k = 0; k < kDim / 8; ++k)
          if (k * 8 < dim)
            *reinterpret_cast<float2*>(to + i * (dim + 4) + k * 8 + 2 * t) = {o[k][2 * h], o[k][2 * h + 1]};
      }
    }
  }
};

// bf16, up to 8 queries, with the tokens (the elements of a value) on a product's 16 rows and the queries
// on its 8 columns: half the products of ManyCore and half its registers, so 12 warps an SM and not 8 (256
// sequences of 0 to 8192 tokens, 8 heads of 128, 4 queries each: 825 us by ManyCore, 682 to 712 so, 6 TB/s).  Registers
// are for 12 warps of 128 elements, not for 16 that the rings leave no room for: 718 us with a spill.
// Lane (g, t) has queries 2t and 2t + 1 of tokens g and g + 8; the weights are transposed into the
// second product's operand.
//   The reference lags, and no maximum is taken while a vote finds all scores below it + kLag: sums cross
// lanes at an item's end only.
template <int kDim_>
struct FewCore {
  using E = __nv_bfloat16;
  static constexpr int kBlk = 16;
  static constexpr int kDim = kDim_, kMostWarps = kDim <= 64 ? 10 : kDim <= 128 ? 12 : 8, kMaxQ = 8;
  static constexpr int kSteps = kDim / 16, kPacks = kDim / 8;
  static constexpr int kScratch = 0;
  uint32_t q[kSteps][2];
  float o[kSteps][4];
  float m[2], l[2];
  int lim[2];

  ALR_DEV void load_q(const KvPass& p, long long row0, int h0, int n_q, int gw, void*) {
    const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3, r = g / p.gw;
    const bool there = g < n_q && g - r * p.gw < gw;
    const E* src = static_cast<const E*>(p.a.Q) +
                   (there ? (row0 + r) * p.a.ldq + (h0 + g - r * p.gw) * p.a.c.dim : 0);
#pragma unroll
    for (int k = 0; k < kSteps; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int d = k * 16 + e * 8 + 2 * t;
        q[k][e] = there && d < p.a.c.dim ? *reinterpret_cast<const uint32_t*>(src + d) : 0u;
      }
  }
  ALR_DEV void zero() {
    m[0] = m[1] = kNoRef;
    l[0] = l[1] = 0.f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  }
  ALR_DEV void see(const KvPass& p, int tokens, int n_q) {
    const int t = threadIdx.x & 3;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int v = __shfl_sync(~0u, tokens, (2 * t + h) / p.gw);
      lim[h] = 2 * t + h < n_q ? v : kNoQuery;
    }
  }
  ALR_DEV void add(const KvPass& p, char* ring, int row_bytes, int t0, uint32_t there, bool plain, void*) {
    const int lane = threadIdx.x & 31, g = lane >> 2;
    const uint32_t at = smem_u32(ring) + (lane & (kBlk - 1)) * row_bytes + (lane >> 4) * 16;
    float s[4] = {}, s2[4] = {};
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      if (k * 16 >= p.a.c.dim) break;
      uint32_t a[4];
      ldmatrix4(a, at + 32 * k);
      mma_16816(k & 1 ? s2 : s, a, q[k][0], q[k][1]);
    }
    const float c = p.a.scale * kLog2e;
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = __fmul_rn(s[e] + s2[e], c);   // never an fma with the reference
    if (!plain) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int tok = g + 8 * (e >> 1);
        if (t0 + tok >= lim[e & 1] || !(there >> tok & 1)) s[e] = kNegInf;
      }
    }
    if (__any_sync(~0u, fmaxf(s[0], s[2]) - m[0] > kLag || fmaxf(s[1], s[3]) - m[1] > kLag)) {
      float f[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float up = fmaxf(s[h], s[h + 2]);
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) up = fmaxf(up, __shfl_xor_sync(~0u, up, off));
        up = fmaxf(m[h], up);
        f[h] = m[h] == up ? 1.f : ex2(m[h] - up);
        m[h] = up;
        l[h] *= f[h];
      }
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        o[i][0] *= f[0], o[i][1] *= f[1];
        o[i][2] *= f[0], o[i][3] *= f[1];
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = ex2(s[e] - m[e & 1]);
    l[0] += s[0] + s[2];
    l[1] += s[1] + s[3];
    // the product's only operand type: a weight is off by 2^-8, l is not
    const uint32_t b0 = transpose8(pack_bf16(s[0], s[1])), b1 = transpose8(pack_bf16(s[2], s[3]));
    const uint32_t vat = smem_u32(ring) + kBlk * row_bytes + (((lane >> 4) << 3) + (lane & 7)) * row_bytes +
                         (lane >> 3 & 1) * 16;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if (i * 16 >= p.a.c.dim) break;
      uint32_t a[4];
      ldmatrix4_t(a, vat + 32 * i);
      mma_16816(o[i], a, b0, b1);
    }
  }
  ALR_DEV void leave(int n_q, int dim, float* to) {
    const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
    float* ml = to + n_q * (dim + 4);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) l[h] += __shfl_xor_sync(~0u, l[h], off);
      const int i = 2 * t + h;
      if (i < n_q) {
        if (g == 0) ml[2 * i] = l[h] == 0.f ? kNegInf : m[h], ml[2 * i + 1] = l[h];
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (k * 16 + e * 8 < dim) to[i * (dim + 4) + k * 16 + e * 8 + g] = o[k][h + 2 * e];
      }
    }
  }
};

// fp32 by fused multiply-adds (a tensor product in tf32 would lose 13 bits of the inputs).  Scores: lane
// (h, i) = (lane / kBlk, lane % kBlk) takes its share of the packs of token i; weights go through shared memory;
// values: a lane owns whole packs of the result, groups of lanes share the tokens where there are
// fewer packs than lanes.  (48 sequences of up to 4001 tokens, 16 heads of 80, one query each: 206 us, 4.8
// TB/s; 32 blocks of 8 rows over 1000 to 3000, 32 heads of 128: 441 us, 19 TFLOP/s.)
template <int kDim_, int kQ>
struct F32Core {
  using E = float;
  // Long rows of several queries in shorter blocks, whose rings leave room for more warps (128 rollouts of a
  // prefix of 4000 tokens, 64 heads on 8 of 256: 1706 us by blocks of 16, 1081 so; 32 blocks of 8 rows, 32
  // heads on 8 of 128: 486 and 441; 48 sequences of up to 3000 tokens, 16 heads on 4 of 256: 135 and 121).
  static constexpr int kBlk = kDim_ > 128 || (kQ == 8 && kDim_ >= 128) ? 8 : 16, kShares = 32 / kBlk;
  static constexpr int kDim = kDim_, kMostWarps = kQ == 1 ? 16 : 8, kMaxQ = kQ;
  static constexpr int kPacks = kDim / 4;
  static constexpr int kOwn = kPacks > 32 ? kPacks / 32 : 1;       // packs of a lane
  static constexpr int kGroups = kPacks < 32 ? 32 / kPacks : 1;    // lanes that share a pack
  static constexpr int kScratch = (kQ * kDim + kBlk * kQ) * 4;     // queries, weights
  float o[kQ][kOwn][4];
  float m[kQ], l[kQ];          // l: of the lane's token
  int lim[kQ];

  ALR_DEV void load_q(const KvPass& p, long long row0, int h0, int n_q, int gw, void* scratch) {
    float* qs = static_cast<float*>(scratch);
    __syncwarp();
#pragma unroll 1
    for (int i = 0; i < kQ; ++i) {
      const int r = i / p.gw;
      const float* src =
          static_cast<const float*>(p.a.Q) + (row0 + r) * p.a.ldq + (h0 + i - r * p.gw) * p.a.c.dim;
      for (int c = threadIdx.x & 31; c < kPacks; c += 32) {
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < n_q && i - r * p.gw < gw && 4 * c < p.a.c.dim) x = *reinterpret_cast<const float4*>(src + 4 * c);
        reinterpret_cast<float4*>(qs + i * kDim)[c] = x;
      }
    }
    __syncwarp();
  }
  ALR_DEV void zero() {
#pragma unroll
    for (int i = 0; i < kQ; ++i) {
      m[i] = kNegInf;
      l[i] = 0.f;
#pragma unroll
      for (int k = 0; k < kOwn; ++k) o[i][k][0] = o[i][k][1] = o[i][k][2] = o[i][k][3] = 0.f;
    }
  }
  ALR_DEV void see(const KvPass& p, int tokens, int n_q) {
#pragma unroll
    for (int i = 0; i < kQ; ++i) lim[i] = __shfl_sync(~0u, tokens, (i / p.gw) & 31);
  }
  ALR_DEV void add(const KvPass& p, const char* ks, int row_bytes, int t0, uint32_t there, bool plain,
                   void* scratch) {
    const char* vs = ks + kBlk * row_bytes;
    const float* qs = static_cast<const float*>(scratch);
    float* ws = static_cast<float*>(scratch) + kQ * kDim;
    const int lane = threadIdx.x & 31, tok = lane % kBlk, share = lane / kBlk;
    const int packs = p.a.c.dim / 4;
    float s[kQ] = {};
#pragma unroll 4
    for (int c = share; c < packs; c += kShares) {
      const float4 k = *reinterpret_cast<const float4*>(ks + tok * row_bytes + 16 * c);
#pragma unroll
      for (int i = 0; i < kQ; ++i) {
        const float4 x = reinterpret_cast<const float4*>(qs + i * kDim)[c];
        s[i] = fmaf(k.x, x.x, fmaf(k.y, x.y, fmaf(k.z, x.z, fmaf(k.w, x.w, s[i]))));
      }
    }
    const float c = p.a.scale * kLog2e;
    const bool here = (there >> tok & 1) != 0;
    bool moves = false;
    float top[kQ];
#pragma unroll
    for (int i = 0; i < kQ; ++i) {
#pragma unroll
      for (int off = kBlk; off < 32; off <<= 1) s[i] += __shfl_xor_sync(~0u, s[i], off);
      s[i] = __fmul_rn(s[i], c);             // never an fma with the reference
      if (!plain && (t0 + tok >= lim[i] || !here)) s[i] = kNegInf;
      top[i] = warp_max(s[i]);
      moves |= top[i] > m[i] + kLag;
    }
    float f[kQ];
#pragma unroll
    for (int i = 0; i < kQ; ++i) f[i] = 1.f;
    if (moves) {                                     // the same in all lanes
#pragma unroll
      for (int i = 0; i < kQ; ++i) {
        const float up = fmaxf(m[i], top[i]);
        f[i] = m[i] == up ? 1.f : ex2(m[i] - up);
        m[i] = up;
        l[i] *= f[i];
#pragma unroll
        for (int k = 0; k < kOwn; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][k][e] *= f[i];
      }
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kQ; ++i) {
      const float e = ex2(s[i] - (m[i] == kNegInf ? 0.f : m[i]));
      if (share == 0) {
        l[i] += e;
        ws[tok * kQ + i] = e;
      }
    }
    __syncwarp();
    const int group = kGroups > 1 ? lane / kPacks : 0, own = kGroups > 1 ? lane % kPacks : lane;
#pragma unroll 4
    for (int j = group; j < kBlk; j += kGroups) {
      float4 v[kOwn];
#pragma unroll
      for (int k = 0; k < kOwn; ++k)
        v[k] = own + 32 * k < packs ? *reinterpret_cast<const float4*>(vs + j * row_bytes + 16 * (own + 32 * k))
                                 : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kQ; ++i) {
        const float e = ws[j * kQ + i];
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
          o[i][k][0] = fmaf(e, v[k].x, o[i][k][0]);
          o[i][k][1] = fmaf(e, v[k].y, o[i][k][1]);
          o[i][k][2] = fmaf(e, v[k].z, o[i][k][2]);
          o[i][k][3] = fmaf(e, v[k].w, o[i][k][3]);
        }
      }
    }
  }
  ALR_DEV void leave(int n_q, int dim, float* to) {
    const int lane = threadIdx.x & 31, own = kGroups > 1 ? lane % kPacks : lane;
    float* ml = to + n_q * (dim + 4);
#pragma unroll
    for (int i = 0; i < kQ; ++i) {
      if (i >= n_q) break;
      const float sum = warp_reduce(l[i], AddOp());
      if (lane == 0) ml[2 * i] = m[i], ml[2 * i + 1] = sum;
#pragma unroll
      for (int k = 0; k < kOwn; ++k) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int off = kPacks; off < 32; off <<= 1) o[i][k][e] += __shfl_xor_sync(~0u, o[i][k][e], off);
        const int d = 4 * (own + 32 * k);
        if (lane < kPacks && d < dim)
          *reinterpret_cast<float4*>(to + i * (dim + 4) + d) =
              make_float4(o[i][k][0], o[i][k][1], o[i][k][2], o[i][k][3]);
      }
    }
  }
};

// ------------------------------------------------------------------------ kernel ---
ALR_DEV void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// Arrive on `bar` once all copies this thread issued so far have landed.
ALR_DEV void cp_async_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
ALR_DEV void put_zeros16(uint32_t dst) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst), "r"(0) : "memory");
}

// Bytes of a token's row in shared memory: its packs of 16 bytes, of bf16 an even number of them (a
// product takes 16 elements), and one more where that makes them odd.
template <typename E>
__host__ __device__ constexpr int row_bytes_of(int dim) {
  const int packs = dim * int(sizeof(E)) / 16, full = sizeof(E) == 2 ? (packs + 1) / 2 * 2 : packs;
  return (full | 1) * 16;
}

constexpr int kMostStages = 8;

// -------------------------------------------------------------------------- join ---
// Partial results of an item.  A query's largest m and the weights of its parts come from the parts'
// scalars, a lane a part; then a warp adds up all or some of the parts, each load independent of
// the others.  The order is the parts', whatever the timing.
constexpr int kJoinWarps = 16;

struct JoinItem {
  long long row0;
  int n_rows, gw, h0, n_q;                   // n_q: queries that exist
  ALR_DEV JoinItem(const KvPass& p, const int4& cut) {
    n_rows = tile_rows(p, cut.x, row0);
    const int group = p.a.H / p.a.c.heads, kv = cut.y / p.gs, slice = (cut.y - kv * p.gs) * p.gw;
    gw = min(p.gw, group - slice);
    h0 = kv * group + slice;
    n_q = n_rows * gw;
  }
  ALR_DEV int query(const KvPass& p, int k, int& r) const {   // place of the k-th
    r = k / gw;
    return r * p.gw + (k - r * gw);
  }
};

struct JoinSums {
  float m = kNegInf, l = 0.f;                // l: to be added over the lanes
  float4 o[2] = {};
};

// Parts 0 to n - 1 of query q: part k in place slot0 + 2 k, but part 0 in slot0 + 1 if `opened`; o of
// those k = sub, sub + share, ...
ALR_DEV void join_parts(const KvPass& p, const float* parts, int slot0, bool opened, int n, int q, int sub,
                        int share, JoinSums& s) {
  const int lane = threadIdx.x & 31, dim = p.a.c.dim;
  const long long stride = part_floats(p.max_q, dim);
  const auto part = [&](int k) { return parts + (slot0 + (k == 0 && opened ? 1 : 2 * k)) * stride; };
  float2 first = {kNegInf, 0.f};
  if (lane < n) {
    first = *reinterpret_cast<const float2*>(part(lane) + p.max_q * dim + 2 * q);
  }
  float m = first.x;
  for (int k = lane + 32; k < n; k += 32) m = fmaxf(m, part(k)[p.max_q * dim + 2 * q]);
  s.m = warp_max(m);
  const float ref = s.m == kNegInf ? 0.f : s.m;
  for (int k0 = 0; k0 < n; k0 += 32) {
    float w = 0.f;
    if (k0 + lane < n) {
      if (k0 > 0) first = *reinterpret_cast<const float2*>(part(k0 + lane) + p.max_q * dim + 2 * q);
      w = first.x == ref ? 1.f : ex2(first.x - ref);
      s.l = fmaf(first.y, w, s.l);
    }
    const int some = min(32, n - k0);
#pragma unroll 4
    for (int k = sub; k < some; k += share) {
      const float f = __shfl_sync(~0u, w, k);
      const float4* x = reinterpret_cast<const float4*>(part(k0 + k) + q * dim);
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (4 * (lane + 32 * e) < dim) {
          const float4 y = x[lane + 32 * e];
          s.o[e] = make_float4(fmaf(y.x, f, s.o[e].x), fmaf(y.y, f, s.o[e].y), fmaf(y.z, f, s.o[e].z),
                               fmaf(y.w, f, s.o[e].w));
        }
    }
  }
}

template <typename E>
ALR_DEV void put_sums(const KvPass& p, const KvRowOut& to, const JoinSums& s) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const float v[4] = {s.o[e].x, s.o[e].y, s.o[e].z, s.o[e].w};
    if (4 * (lane + 32 * e) < p.a.c.dim) put<E, 4>(to, 4 * (lane + 32 * e), v);
  }
}

// Each warp is a worker with a ring of its own: no block-wide barrier after the start, so warps in
// different items never wait for one another, and a ring's blocks (all but one ahead) are all that
// hides latency.  Long sequences run near the memory's rate; short ones are latency, the chain of lengths,
// table, keys, results and join (64 sequences of up to 1024 tokens: 62 us cold for 134 MB).
//   Copies are of 16 bytes: bulk copies of a row each took 1020 us where these took 830.
template <typename Core>
__global__ void __launch_bounds__(Core::kMostWarps * 32, 1)
    kv_blocks_kernel(const __grid_constant__ KvPass p, int* status) {
  using E = typename Core::E;
  constexpr int kBlk = Core::kBlk, kPacks = Core::kPacks, kPack = 16 / sizeof(E);
  constexpr uint32_t kAll = (1u << kBlk) - 1;
  constexpr int kRowsAt = 32 / kPacks > 1 ? 32 / kPacks : 1;      // rows of one copy instruction
  constexpr int kCopies = kBlk * kPacks / 32;
  extern __shared__ __align__(128) char ring_smem[];
  __shared__ WorkerStart starts[Core::kMostWarps + 1];
  __shared__ long long buf[Core::kMostWarps];
  __shared__ uint32_t there_of[Core::kMostWarps][kMostStages];
  __shared__ uint64_t landed[Core::kMostWarps][kMostStages];
  __shared__ KvRowOut outs[Core::kMostWarps][Core::kMaxQ];
  __shared__ int4 cut_of[Core::kMostWarps];  // (tile, unit, parts) of the item that a worker leaves open
  __shared__ int4 head_cut;                  // ... of the item that the block's first worker continues
  __shared__ int abort_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const KvAttention& a = p.a;
  const int stages = p.stages, row_bytes = row_bytes_of<E>(a.c.dim), slot_bytes = 2 * kBlk * row_bytes;
  char* ring = ring_smem + warp * (stages * slot_bytes + Core::kScratch);
  void* scratch = ring + stages * slot_bytes;
  if (lane == 0) {
    for (int i = 0; i < stages; ++i)         // one more than ever comes: withheld
      mbar_init(&landed[warp][i], 32 + (i == 0 && a.withhold_first_stage ? 1 : 0));
    fence_mbar_init();
  }
  if (threadIdx.x == 0) {
    abort_word = 0;
    head_cut = make_int4(0, 0, 0, 0);
  }
  if (lane == 0) cut_of[warp] = make_int4(0, 0, 0, 0);
  const AbortFlag ab{&abort_word, status};
  pdl_wait();
  const Line line = p.one_each ? find_item_starts<kBlk>(p, starts, buf)
                               : find_starts<kBlk>(p, starts, reinterpret_cast<long long*>(ring_smem), buf);
  if (a.c.dim % 16 != 0)                     // what lies past a row's end is never copied: zeros
    for (int i = lane; i < stages * slot_bytes / 16; i += 32)
      reinterpret_cast<uint4*>(ring)[i] = make_uint4(0, 0, 0, 0);
  // this warp among all workers (its places for partial results), and on the line
  const int id0 = blockIdx.x * (p.one_each ? p.block_workers : line.per_block), id = id0 + warp;
  const int on_line = p.one_each ? warp : id;
  const bool works = warp < line.per_block && on_line < line.n;
  const int count = works ? int(starts[warp + 1].block - starts[warp].block) : 0;
  Cursor<kBlk> in{};                         // of the loads
  if (count > 0) in.start(p, starts[warp].tile, starts[warp].unit, starts[warp].b);
  Cursor<kBlk> at = in;                      // of the sums

  // page and position in it of the lane's token (lane % kBlk) in the next block to load
  int j = 0, off = 0, pg = -1;
  const auto look_up = [&](bool runs_on) {
    if (runs_on) {
      j += p.step_pg;
      off += p.step_tok;
      if (off >= a.c.page) off -= a.c.page, ++j;
    } else {
      const int tok = in.t0 + (lane & (kBlk - 1));
      j = tok / a.c.page;
      off = tok - j * a.c.page;
    }
    pg = in.t0 + (lane & (kBlk - 1)) < in.most ? a.table[(long long)in.seq * a.cols + j] : -1;
  };
  if (count > 0) look_up(false);
  const uint32_t ring_at = smem_u32(ring);
  const bool block_in_page = a.c.page % kBlk == 0;
  const int pack = lane % kPacks, sub = kPacks < 32 ? lane / kPacks : 0;
  long long head = (long long)(in.unit / p.gs) * a.c.sh + pack * kPack;      // of the next block
  const auto load = [&](int slot) {
    const bool there = pg >= 0 && pg < a.c.n_pages;
    const uint32_t all = __ballot_sync(~0u, there) & kAll;
    if (lane == 0) there_of[warp][slot] = all;
    const E* K = static_cast<const E*>(a.c.K) + head;
    const E* V = static_cast<const E*>(a.c.V) + head;
    const uint32_t dst = ring_at + slot * slot_bytes + pack * 16, v_off = kBlk * row_bytes;
    if (block_in_page && all == kAll) {
      // one page: rows a fixed step apart
      const long long from = pg * a.c.sp + (off - (lane & (kBlk - 1)) + sub) * a.c.st;
      const E* k = K + from;
      const E* v = V + from;
      uint32_t to = dst + sub * row_bytes;
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        constexpr int kSame = kPacks > 32 ? kPacks / 32 : 1;         // instructions of one row
        const int cc = i % kSame * 32;
        if ((pack + cc) * kPack < a.c.dim) {
          cp_async16(to + cc * 16, k + cc * kPack);
          cp_async16(to + v_off + cc * 16, v + cc * kPack);
        }
        if (i % kSame == kSame - 1) {
          k += kRowsAt * a.c.st;
          v += kRowsAt * a.c.st;
          to += kRowsAt * row_bytes;
        }
      }
    } else {
      const long long row = there ? pg * a.c.sp + off * a.c.st : 0;
#pragma unroll 4
      for (int i = 0; i < kCopies; ++i) {
        constexpr int kSame = kPacks > 32 ? kPacks / 32 : 1;
        const int cc = i % kSame * 32, r = i / kSame * kRowsAt + sub;
        const long long from = __shfl_sync(~0u, row, r) + cc * kPack;
        if ((pack + cc) * kPack < a.c.dim) {
          const uint32_t to = dst + r * row_bytes + cc * 16;
          if (all >> r & 1) {
            cp_async16(to, K + from);
            cp_async16(to + v_off, V + from);
          } else {                           // weights of 0 meet zeros
            put_zeros16(to);
            put_zeros16(to + v_off);
          }
        }
      }
    }
    cp_async_arrive(&landed[warp][slot]);
  };
  int loaded = 0, load_slot = 0, slot = 0;
  uint32_t round = 0;
  const auto load_next = [&]() {
    if (loaded < count) {
      load(load_slot);
      if (++load_slot == stages) load_slot = 0;
      if (++loaded < count) {
        const bool on = in.advance(p);
        if (!on) head = (long long)(in.unit / p.gs) * a.c.sh + pack * kPack;
        look_up(on);
      }
    }
  };
  __syncwarp();
  for (int i = 0; i < stages - 1; ++i) load_next();

  Core core;
  int i = 0;
  while (i < count) {
    // an item, or what the stretch has of it
    long long row0;
    const int n_rows = max(tile_rows(p, at.tile, row0), 0);
    const int group = a.H / a.c.heads, kv = at.unit / p.gs, slice = (at.unit - kv * p.gs) * p.gw;
    const int gw = min(p.gw, group - slice), h0 = kv * group + slice, n_q = n_rows * p.gw;
    const Tile tile = at.t;
    const int b0 = at.b, b1 = min(tile.nb, b0 + (count - i));
    core.load_q(p, row0, h0, n_q, gw, scratch);
    core.zero();
    const bool last_here = b1 == tile.nb;
    const int tile_id = at.tile, unit = at.unit;
    bool on = false;
    int least = 0;                               // tokens of the run that all rows see
    for (int b = b0; b < b1; ++b, ++i) {
      if (!on) {
        const int tokens = at.lead >= 0 && tile.lead == at.lead ? tile.len : 0;
        least = warp_min(lane < n_rows ? tokens : INT_MAX);
        core.see(p, tokens, n_q);
      }
      wait_on(&landed[warp][slot], round, ab);
      __syncwarp();                              // all lanes are done with the slot that is filled next
      load_next();
      const uint32_t there = there_of[warp][slot];
      core.add(p, ring + slot * slot_bytes, row_bytes, at.t0, there,
               least - at.t0 >= kBlk && there == kAll, scratch);
      if (++slot == stages) slot = 0, ++round;
      if (i + 1 < count) on = at.advance(p);
    }
    const bool whole = b0 == 0 && last_here, opens = b0 == 0 && !last_here;
    const int part = 2 * id + (opens ? 1 : 0);
    const auto out = [&](int q, int r, float m, float l, bool writer) {
      return whole ? row_out(p, row0 + r, h0 + q - r * p.gw, m, l, writer)
                   : part_out(p, p.parts, part, q, m, l, writer);
    };
    // through the slot just used, which is filled again only in the next block's turn, into whole packs
    const int dim = a.c.dim, used = slot == 0 ? stages - 1 : slot - 1;
    float* sums = reinterpret_cast<float*>(ring + used * slot_bytes);
    __syncwarp();
    core.leave(n_q, dim, sums);
    __syncwarp();
    const float* ml = sums + n_q * (dim + 4);
    if (lane < n_q) {
      const int r = lane / p.gw;
      KvRowOut to = {0.f, 0.f, nullptr, nullptr, nullptr};
      if (lane - r * p.gw < gw) to = out(lane, r, ml[2 * lane], ml[2 * lane + 1], true);
      outs[warp][lane] = to;
    }
    __syncwarp();
    float odd = lane < n_q ? ml[2 * lane + 1] * 0.f : 0.f;         // 0 while all values are finite
    const int quads = dim / 4;
#pragma unroll 2
    for (int k = lane; k < n_q * quads; k += 32) {
      const int q = k / quads, d = 4 * (k - q * quads);
      const KvRowOut to = outs[warp][q];
      const float4 x = *reinterpret_cast<const float4*>(sums + q * (dim + 4) + d);
      const float v[4] = {x.x, x.y, x.z, x.w};
      if (to.dst != nullptr || to.dst_f != nullptr) put<E, 4>(to, d, v);
      odd = fmaf(0.f, (x.x + x.y) + (x.z + x.w), odd);
    }
    if (__any_sync(~0u, !(odd == 0.f))) {
#pragma unroll 1
      for (int q = 0; q < n_q; ++q) {
        const int r = q / p.gw;
        const float sum = ml[2 * q + 1];         // NaN: of its own scores, and so are its results
        if (q - r * p.gw >= gw || sum != sum) continue;
        int seq, t0, t1;
        row_tokens<kBlk>(tile, r, b0, b1, seq, t0, t1);
        __syncwarp();
        take_again<E, Core::kDim, 1>(p, row0 + r, h0 + q - r * p.gw, seq, t0, t1, whole ? nullptr : p.parts, part, q);
      }
    }
    __syncwarp();
    if (dim % 16 != 0) {                         // zeros past the rows' ends again
      for (int k = lane; k < slot_bytes / 16; k += 32) reinterpret_cast<uint4*>(sums)[k] = make_uint4(0, 0, 0, 0);
      __syncwarp();
    }
    if (!whole && lane == 0) {
      const int parts = last_here ? 1 : line.last_before(line.start(on_line + 1) + (tile.nb - b1)) - on_line + 1;
      if (opens) cut_of[warp] = make_int4(tile_id, unit, parts, 0);
      else if (warp == 0) head_cut = make_int4(tile_id, unit, parts, 0);
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  // ---- the items that the block's workers share: a warp a query
  int4 cut = make_int4(0, 0, 0, 0);
  int turn = 0;
  for (int w = -1; w < line.per_block; ++w) {
    const int4 c = w < 0 ? head_cut : cut_of[w];
    if (c.z == 0) continue;
    const JoinItem t(p, c);
    const int from = w < 0 ? 0 : w, here = min(c.z, line.per_block - from), slot0 = 2 * (id0 + from);
    const bool inside = w >= 0 && c.z == here;
    const int to_slot = 2 * blockIdx.x + (w < 0 ? 0 : 1);
    if (w >= 0 && !inside)
      cut = make_int4(c.x, c.y, (id0 + w + c.z - 1) / line.per_block - int(blockIdx.x) + 1, 0);
    for (int k = 0; k < t.n_q; ++k, ++turn) {
      if (turn % (blockDim.x / 32) != warp) continue;
      int r;
      const int q = t.query(p, k, r);
      JoinSums s;
      join_parts(p, p.parts, slot0, w >= 0, here, q, 0, 1, s);
      const float l = warp_reduce(s.l, AddOp());
      const KvRowOut o = inside ? row_out(p, t.row0 + r, t.h0 + q - r * p.gw, s.m, l, lane == 0)
                                : part_out(p, p.block_parts, to_slot, q, s.m, l, lane == 0);
      put_sums<E>(p, o, s);
    }
  }
  if (threadIdx.x == 0 && !p.one_each) p.cuts[blockIdx.x] = cut;
  pdl_release();
}

// --------------------------------------------------- join of items across blocks ---
template <typename E>
__global__ void __launch_bounds__(kJoinWarps * 32, 3) kv_join_kernel(const __grid_constant__ KvPass p) {
  __shared__ float4 sums[kJoinWarps][kKvMaxDim / 4];
  pdl_wait_and_release();
  const int id = blockIdx.x;
  const int4 cut = p.cuts[id];
  if (cut.z == 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, dim = p.a.c.dim;
  const JoinItem t(p, cut);
  const int q_first = blockIdx.y * kJoinWarps, n_q = min(t.n_q - q_first, kJoinWarps);
  if (n_q <= 0) return;
  const int share = kJoinWarps / n_q, sub = warp % share;            // warps of a query
  if (warp >= n_q * share) return;
  int r;
  const int q = t.query(p, q_first + warp / share, r);
  JoinSums s;
  join_parts(p, p.block_parts, 2 * id, true, cut.z, q, sub, share, s);
  const float l = warp_reduce(s.l, AddOp());
  if (share > 1) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (4 * (lane + 32 * e) < dim) sums[warp][lane + 32 * e] = s.o[e];
    named_bar_sync(1 + warp / share, share * 32);
    if (sub != 0) return;
    for (int k = 1; k < share; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (4 * (lane + 32 * e) < dim) {
          const float4 y = sums[warp + k][lane + 32 * e];
          s.o[e] = make_float4(s.o[e].x + y.x, s.o[e].y + y.y, s.o[e].z + y.z, s.o[e].w + y.w);
        }
  }
  put_sums<E>(p, row_out(p, t.row0 + r, t.h0 + q - r * p.gw, s.m, l, lane == 0), s);
}

// ---------------------------------------------------------------------- launches ---
constexpr int kRingsMost = 218 * 1024;       // bytes of all rings of a block

template <typename E>
cudaError_t run_join(const KvPass& p, int sms, cudaStream_t s) {
  const dim3 grid(std::min(sms, kKvMostSms), (p.max_q + kJoinWarps - 1) / kJoinWarps);
  return launch_pdl(kv_join_kernel<E>, grid, dim3(kJoinWarps * 32), 0, s, p);
}

template <typename Core>
cudaError_t run_pass(KvPass p, int sms, int* status, cudaStream_t s) {
  using E = typename Core::E;
  constexpr int kBlk = Core::kBlk;
  shape_pass(p, Core::kMaxQ, 32, kBlk);
  // as many warps as have two blocks each, then as many blocks
  const int slot = 2 * kBlk * row_bytes_of<E>(p.a.c.dim);
  const int warps = std::min(Core::kMostWarps, kRingsMost / (2 * slot + Core::kScratch));
  p.stages = std::min(kMostStages, (kRingsMost / warps - Core::kScratch) / slot);
  // Few items of few blocks: each its own thread block, nothing to share out or to join (12 sequences of up
  // to 60 tokens, 5 heads: 17.7 us in even stretches and a join, 13.5 so).
  const long long items = (long long)p.n_tiles * p.n_units;
  const long long most = (long long)p.a.cols * p.a.c.page;             // tokens of a row
  p.one_each = items <= std::min(sms, kKvMostSms) && (most + kBlk - 1) / kBlk * p.rows <= 4 * warps;
  const int grid = p.one_each ? int(items) : std::min(sms, kKvMostSms);
  const int ring = warps * (p.stages * slot + Core::kScratch);
  p.block_workers = warps;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_smem(kv_blocks_kernel<Core>, kRingsMost, done);
  if (e != cudaSuccess) return e;
  const cudaError_t f = launch_pdl(kv_blocks_kernel<Core>, dim3(grid), dim3(warps * 32), ring, s, p, status);
  return f != cudaSuccess || p.one_each ? f : run_join<E>(p, sms, s);
}

template <int kDim>
cudaError_t run_f32(const KvPass& p, int sms, int* status, cudaStream_t s) {
  const long long q = std::min<long long>(p.part.per, p.a.N) * (p.a.H / p.a.c.heads);
  return q <= 1   ? run_pass<F32Core<kDim, 1>>(p, sms, status, s)
         : q <= 4 ? run_pass<F32Core<kDim, 4>>(p, sms, status, s)
                  : run_pass<F32Core<kDim, 8>>(p, sms, status, s);
}

template <int kDim>
cudaError_t run_dim(const KvPass& p, int sms, int* status, cudaStream_t s) {
  if (p.a.c.dtype != 0) return run_f32<kDim>(p, sms, status, s);
  const long long q = std::min<long long>(p.part.per, p.a.N) * (p.a.H / p.a.c.heads);
  return q <= 8 ? run_pass<FewCore<kDim>>(p, sms, status, s) : run_pass<ManyCore<kDim>>(p, sms, status, s);
}

// More queries of the same tokens than one warp holds: tiles by tcgen05.
bool takes_tiles(const KvAttention& a, int rows) {
  return a.c.dtype == 0 && a.c.dim <= 128 && std::min<long long>(rows, a.N) * (a.H / a.c.heads) > 16 &&
         a.c.n_pages > 0 && a.scale >= 0.f;
}

cudaError_t run_part(KvPass p, const KvMaps& maps, int sms, int* status, cudaStream_t s) {
  const int dim = p.a.c.dim;
  if (takes_tiles(p.a, p.part.per)) {
    const cudaError_t e = launch_kv_tc(p, maps, sms, status, s);
    return e != cudaSuccess ? e : run_join<__nv_bfloat16>(p, sms, s);
  }
  if (p.a.c.dtype != 0 && dim <= 32) return run_f32<32>(p, sms, status, s);   // bf16: no faster than by 64
  return dim <= 64    ? run_dim<64>(p, sms, status, s)
         : dim <= 128 ? run_dim<128>(p, sms, status, s)
                      : run_dim<256>(p, sms, status, s);
}

size_t up16(size_t x) { return (x + 15) / 16 * 16; }

struct Layout {
  size_t parts, block_parts, cuts, pre_o, pre_ml, total;
};

Layout layout(long long N, int H, int dim, bool prefix) {
  Layout y;
  size_t at = 0;
  y.parts = at;                              // 16 workers of 8 queries or 8 of 16 an SM
  at += size_t(2 * 16 * kKvMostSms) * 8 * (dim + 4) * sizeof(float);
  y.block_parts = at;                        // 128 queries at most
  at += size_t(2 * kKvMostSms) * 128 * (dim + 4) * sizeof(float);
  y.cuts = at;
  at += size_t(kKvMostSms) * sizeof(int4);
  y.pre_o = at;
  if (prefix) at += up16(size_t(N) * H * dim * sizeof(float));
  y.pre_ml = at;
  if (prefix) at += up16(size_t(N) * H * 2 * sizeof(float));
  y.total = at;
  return y;
}

}  // namespace

size_t kv_attention_workspace(long long N, int H, int dim, bool prefix) {
  return layout(N, H, dim, prefix).total;
}

bool kv_attention_takes_maps(const KvAttention& a, int rows) {
  return takes_tiles(a, rows) && a.c.dim % 16 == 0;
}

cudaError_t launch_kv_attention(const KvAttention& a, const KvMaps& maps, int sms, int* status,
                                cudaStream_t s) {
  const Layout y = layout(a.N, a.H, a.c.dim, a.prefix_len != nullptr);
  char* ws = static_cast<char*>(a.ws);
  KvPass p{};
  p.a = a;
  p.parts = reinterpret_cast<float*>(ws + y.parts);
  p.block_parts = reinterpret_cast<float*>(ws + y.block_parts);
  p.cuts = reinterpret_cast<int4*>(ws + y.cuts);
  if (a.prefix_len != nullptr) {
    KvPass f = p;
    f.part = {a.prefix_seq, a.prefix_len, a.rows_per_prefix};
    f.put_o = reinterpret_cast<float*>(ws + y.pre_o);
    f.put_ml = reinterpret_cast<float*>(ws + y.pre_ml);
    const cudaError_t e = run_part(f, maps, sms, status, s);
    if (e != cudaSuccess) return e;
    p.pre_o = f.put_o;
    p.pre_ml = f.put_ml;
    p.a.withhold_first_stage = 0;
  }
  p.part = {a.seq, a.len, a.rows_per_seq};
  return run_part(p, maps, sms, status, s);
}

}  // namespace alr
