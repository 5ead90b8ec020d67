// Attention of query rows over the paged key-value cache, up to 16 queries of a tile at a time.
#include <algorithm>

#include "launch.h"
#include "kv_tiles.cuh"

namespace alr {
namespace {

constexpr int kBlk = 16;       // tokens of a block

// ------------------------------------------------------------------------- cores ---
// A core holds the sums of an item's queries for a warp: load_q, zero, add (one block from the ring, with
// each query's count of visible tokens), finish.
//   Shared memory rows of kDim elements in packs of 16 bytes; pack c of row r lies at place c ^ r
// (of the lowest bits), so that eight rows' packs c fall in different banks.
template <int kPacks>
ALR_DEV int pack_at(int row, int c) {
  return row * kPacks + (kPacks >= 8 ? c ^ (row & 7) : c ^ ((row / (8 / kPacks)) & (kPacks - 1)));
}

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
//   A group of 4 queries leaves 12 rows unused, yet the products are far from the bound: 16 tokens of
// 128 elements are 32 instructions and 8 KB.
template <int kDim_>
struct Bf16Core {
  using E = __nv_bfloat16;
  static constexpr int kDim = kDim_, kWarps = kDim <= 128 ? 8 : 4, kMaxQ = 16;
  static constexpr int kSteps = kDim / 16, kPacks = kDim / 8;
  static constexpr int kStages = kDim <= 32 ? 8 : kDim <= 64 ? 5 : 3;   // blocks of a worker's ring
  static constexpr int kScratch = 0;
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
      const E* src = static_cast<const E*>(p.a.Q) + (there ? (row0 + r) * p.a.ldq + (h0 + i - r * p.gw) * p.a.c.dim : 0);
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
  // lim: visible tokens of the block for the lane's two queries; there: tokens whose page exists.
  ALR_DEV void add(const KvPass& p, uint32_t k_at, uint32_t v_at, const int (&lim)[2], uint32_t there,
                   void*) {
    const int lane = threadIdx.x & 31, t = lane & 3;
    float s[2][4] = {};
    {
      const int row = (lane >> 4) * 8 + (lane & 7), c = lane >> 3 & 1;
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        if (k * 16 >= p.a.c.dim) break;
        uint32_t b[4];
        ldmatrix4(b, k_at + 16 * pack_at<kPacks>(row, 2 * k + c));
        mma_16816(s[0], q[k], b[0], b[1]);
        mma_16816(s[1], q[k], b[2], b[3]);
      }
    }
    const float c = p.a.scale * kLog2e;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] = __fmul_rn(s[n][e], c);   // never an fma with the reference
    if (!__all_sync(~0u, lim[0] >= kBlk && lim[1] >= kBlk && there == 0xffffu)) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int tok = n * 8 + 2 * t + (e & 1);
          if (tok >= lim[e >> 1] || !(there >> tok & 1)) s[n][e] = kNegInf;
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
      ldmatrix4_t(b, v_at + 16 * pack_at<kPacks>(row, 2 * i + c2));
      mma_16816(o[2 * i], w, b[0], b[1]);
      mma_16816(o[2 * i + 1], w, b[2], b[3]);
    }
  }
  // Whether query `half` of the lane got a value that is not finite.
  ALR_DEV bool odd(int half) const {
    float x = l[half];
#pragma unroll
    for (int i = 0; i < kDim / 8; ++i) x = fmaf(0.f, o[i][2 * half] + o[i][2 * half + 1], x);
    return !(x - x == 0.f);
  }
  template <typename Out>
  ALR_DEV uint32_t finish(const KvPass& p, int n_q, void*, Out out) {
    const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
    uint32_t bad = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      l[h] += __shfl_xor_sync(~0u, l[h], 1);
      l[h] += __shfl_xor_sync(~0u, l[h], 2);
      const int i = g + 8 * h;
      const uint32_t who = __ballot_sync(~0u, i < n_q && odd(h));
      for (int k = 0; k < 8; ++k)
        if (who >> (4 * k) & 15u) bad |= 1u << (k + 8 * h);
      if (i >= n_q) continue;
      const KvRowOut r = out(i, m[h], l[h], t == 0);
#pragma unroll
      for (int k = 0; k < kDim / 8; ++k) {
        const int d = k * 8 + 2 * t;
        const float v[2] = {o[k][2 * h], o[k][2 * h + 1]};
        if (d < p.a.c.dim) put<E, 2>(r, d, v);
      }
    }
    return bad;
  }
};

// fp32 by fused multiply-adds (a tensor product in tf32 would lose 13 bits of the inputs).  Scores: lane
// (h, i) = (lane / 16, lane % 16) takes half the packs of token i; weights go through shared memory;
// values: a lane owns whole packs of the result, groups of lanes share the tokens where there are
// fewer packs than lanes.
template <int kDim_, int kQ>
struct F32Core {
  using E = float;
  static constexpr int kDim = kDim_, kWarps = kDim <= 64 ? 8 : kDim <= 128 ? 4 : 2, kMaxQ = kQ;
  static constexpr int kStages = kDim <= 32 ? 5 : 3;
  static constexpr int kPacks = kDim / 4;
  static constexpr int kOwn = kPacks > 32 ? kPacks / 32 : 1;       // packs of a lane
  static constexpr int kGroups = kPacks < 32 ? 32 / kPacks : 1;    // lanes that share a pack
  static constexpr int kScratch = (kQ * kDim + kBlk * kQ) * 4;     // queries, weights
  float o[kQ][kOwn][4];
  float m[kQ], l[kQ];          // l: of the lane's token

  ALR_DEV void load_q(const KvPass& p, long long row0, int h0, int n_q, int gw, void* scratch) {
    float* qs = static_cast<float*>(scratch);
    __syncwarp();
#pragma unroll 1
    for (int i = 0; i < kQ; ++i) {
      const int r = i / p.gw;
      const float* src = static_cast<const float*>(p.a.Q) + (row0 + r) * p.a.ldq + (h0 + i - r * p.gw) * p.a.c.dim;
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
  ALR_DEV void add(const KvPass& p, const char* ks, const char* vs, const int (&lim)[kQ], uint32_t there,
                   void* scratch) {
    const float* qs = static_cast<const float*>(scratch);
    float* ws = static_cast<float*>(scratch) + kQ * kDim;
    const int lane = threadIdx.x & 31, tok = lane & 15, half = lane >> 4;
    const int packs = p.a.c.dim / 4;
    float s[kQ] = {};
#pragma unroll 4
    for (int c = half; c < packs; c += 2) {
      const float4 k = reinterpret_cast<const float4*>(ks)[pack_at<kPacks>(tok, c)];
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
      s[i] = __fmul_rn(s[i] + __shfl_xor_sync(~0u, s[i], 16), c);    // never an fma with the reference
      if (tok >= lim[i] || !here) s[i] = kNegInf;
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
      if (half == 0) {
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
        v[k] = reinterpret_cast<const float4*>(vs)[pack_at<kPacks>(j, own + 32 * k)];
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
  template <typename Out>
  ALR_DEV uint32_t finish(const KvPass& p, int n_q, void*, Out out) {
    const int lane = threadIdx.x & 31;
    const int own = kGroups > 1 ? lane % kPacks : lane;
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < kQ; ++i) {
      if (i >= n_q) break;
      const float sum = warp_reduce(l[i], AddOp());
      float x = sum;
#pragma unroll
      for (int k = 0; k < kOwn; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
          for (int off = kPacks; off < 32; off <<= 1) o[i][k][e] += __shfl_xor_sync(~0u, o[i][k][e], off);
          x = fmaf(0.f, o[i][k][e], x);
        }
      if (__any_sync(~0u, !(x - x == 0.f))) bad |= 1u << i;
      const KvRowOut r = out(i, m[i], sum, lane == 0);
#pragma unroll
      for (int k = 0; k < kOwn; ++k) {
        const int d = 4 * (own + 32 * k);
        if (lane < kPacks && d < p.a.c.dim) put<E, 4>(r, d, o[i][k]);
      }
    }
    return bad;
  }
};

// ------------------------------------------------------------------------ kernel ---
ALR_DEV void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
ALR_DEV void put_zeros16(uint32_t dst) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst), "r"(0) : "memory");
}

// Each warp is a worker with a ring of its own: no block-wide barrier after the start, so warps in
// different items never wait for one another, and a ring's blocks (all but one ahead) are all that
// hides latency: 128 KB of an SM's shared memory in flight.
template <typename Core>
__global__ void __launch_bounds__(Core::kWarps * 32, 1) kv_blocks_kernel(const KvPass p) {
  using E = typename Core::E;
  constexpr int kWarps = Core::kWarps, kStages = Core::kStages, kPacks = Core::kPacks, kPack = 16 / sizeof(E);
  constexpr int kHalf = kBlk * kPacks * 16, kSlot = 2 * kHalf;
  constexpr int kRowsAt = 32 / kPacks > 1 ? 32 / kPacks : 1;      // rows of one copy instruction
  constexpr int kCopies = kBlk * kPacks / 32;
  extern __shared__ __align__(128) char ring_smem[];
  __shared__ WorkerStart starts[kWarps];
  __shared__ long long buf[kWarps];
  __shared__ uint32_t there_of[kWarps][kStages];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  char* ring = ring_smem + warp * (kStages * kSlot + Core::kScratch);
  void* scratch = ring + kStages * kSlot;
  const KvAttention& a = p.a;
  if (a.c.dim != Core::kDim) {               // what lies past a row's end is never copied: zeros
    for (int i = lane; i < kStages * kSlot / 16; i += 32)
      reinterpret_cast<uint4*>(ring)[i] = make_uint4(0, 0, 0, 0);
  }
  pdl_wait();
  const long long total = find_starts<kBlk, kWarps, kWarps>(p, starts, buf);
  const int n = int(min((long long)p.workers, total));
  const int id = warp * gridDim.x + blockIdx.x;
  if (id >= n) {
    if (id < p.workers && lane == 0) p.cuts[id] = make_int4(0, 0, 0, 0);
    pdl_release();
    return;
  }
  const long long begin = stretch(total, n, id), end = stretch(total, n, id + 1);
  Cursor<kBlk> in;                                // of the loads
  in.start(p, starts[warp].tile, starts[warp].rest);
  Cursor<kBlk> at = in;                           // of the sums

  // page and position in it of the lane's token (lane % 16) in the next block to load
  int j = 0, off = 0, pg = -1;
  const auto look_up = [&](bool runs_on) {
    if (runs_on) {
      j += p.step_pg;
      off += p.step_tok;
      if (off >= a.c.page) off -= a.c.page, ++j;
    } else {
      const int tok = in.t0 + (lane & 15);
      j = tok / a.c.page;
      off = tok - j * a.c.page;
    }
    pg = in.t0 + (lane & 15) < in.most ? a.table[(long long)in.seq * a.cols + j] : -1;
  };
  look_up(false);
  const uint32_t ring_at = smem_u32(ring);
  const auto load = [&](int slot) {
    const bool there = pg >= 0 && pg < a.c.n_pages;
    const uint32_t all = __ballot_sync(~0u, there) & 0xffffu;
    if (lane == 0) there_of[warp][slot] = all;
    const long long row = there ? pg * a.c.sp + off * a.c.st : 0;
    const int c = lane % kPacks;
    const long long head = (long long)(in.unit / p.gs) * a.c.sh + c * kPack;
    const E* K = static_cast<const E*>(a.c.K) + head;
    const E* V = static_cast<const E*>(a.c.V) + head;
    const uint32_t dst = ring_at + slot * kSlot;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      int r, cc = c;
      if constexpr (kPacks <= 32) r = i * kRowsAt + lane / kPacks;
      else r = i / (kPacks / 32), cc = c + i % (kPacks / 32) * 32;
      const long long from = __shfl_sync(~0u, row, r) + (cc - c) * kPack;
      if (cc * kPack < a.c.dim) {
        const uint32_t to = dst + 16 * pack_at<kPacks>(r, cc);
        if (all >> r & 1) {
          cp_async16(to, K + from);
          cp_async16(to + kHalf, V + from);
        } else {                             // weights of 0 meet zeros
          put_zeros16(to);
          put_zeros16(to + kHalf);
        }
      }
    }
  };
  const long long count = end - begin;
  long long loaded = 0;
  const auto load_next = [&]() {
    if (loaded < count) {
      load(int(loaded % kStages));
      if (++loaded < count) look_up(in.advance(p));
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  __syncwarp();
  for (int i = 0; i < kStages - 1; ++i) load_next();

  Core core;
  int4 cut = make_int4(0, 0, 0, 0);
  long long i = 0;
  while (i < count) {
    // an item, or what the stretch has of it
    long long row0;
    const int n_rows = tile_rows(p, at.tile, row0);
    const int group = a.H / a.c.heads, kv = at.unit / p.gs, slice = (at.unit - kv * p.gs) * p.gw;
    const int gw = min(p.gw, group - slice), h0 = kv * group + slice;
    const int n_q = max(n_rows, 0) * p.gw;
    const int b0 = at.b, b1 = int(min((long long)at.t.nb, b0 + (count - i)));
    const auto query = [&](int q, int& r) {      // row of query q; whether its head exists
      r = q / p.gw;
      return q < n_q && q - r * p.gw < gw;
    };
    core.load_q(p, row0, h0, n_q, gw, scratch);
    core.zero();
    const bool last_here = b1 == at.t.nb;
    const Tile tile = at.t;
    const long long tile_id = at.tile;
    const int unit = at.unit;
    for (int b = b0; b < b1; ++b, ++i) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
      __syncwarp();
      const int slot = int(i % kStages);
      load_next();
      const uint32_t there = there_of[warp][slot];
      // tokens of the block that each query sees
      const int left = at.lead < 0 || tile.lead != at.lead ? 0 : tile.len - at.t0;
      if constexpr (sizeof(E) == 2) {
        const int g = lane >> 2;
        int lim[2];
        lim[0] = __shfl_sync(~0u, left, (g / p.gw) & 31);
        lim[1] = __shfl_sync(~0u, left, ((g + 8) / p.gw) & 31);
        if (g >= n_q) lim[0] = kBlk;
        if (g + 8 >= n_q) lim[1] = kBlk;
        core.add(p, ring_at + slot * kSlot, ring_at + slot * kSlot + kHalf, lim, there, scratch);
      } else {
        int lim[Core::kMaxQ];
#pragma unroll
        for (int q = 0; q < Core::kMaxQ; ++q) lim[q] = __shfl_sync(~0u, left, (q / p.gw) & 31);
        core.add(p, ring + slot * kSlot, ring + slot * kSlot + kHalf, lim, there, scratch);
      }
      if (i + 1 < count) at.advance(p);
    }
    const bool whole = b0 == 0 && last_here;
    const bool opens = b0 == 0 && !last_here;
    const long long part = 2ll * id + (opens ? 1 : 0);
    const auto out = [&](int q, float m, float l, bool writer) {
      int r;
      if (!query(q, r)) return part_out(p, 2ll * p.workers, 0, m, l, writer);   // nowhere: a spare slot
      return whole ? row_out(p, row0 + r, h0 + q - r * p.gw, m, l, writer)
                   : part_out(p, part, q, m, l, writer);
    };
    uint32_t bad = core.finish(p, n_q, scratch, out);
    if (n_rows > 1 && bad != 0) {
      // Weights of 0 times a value that is not finite: such a value may lie in a token that the query
      // does not see but another of the tile does.  Its tokens again, one by one.
      for (int q = 0; q < n_q; ++q) {
        int r;
        if (!(bad >> q & 1) || !query(q, r)) continue;
        __syncwarp();
        float x[kLaneDims], o[kLaneDims] = {}, m = kNegInf, l = 0.f;
#pragma unroll
        for (int e = 0; e < kLaneDims; ++e)
          x[e] = e * 32 + lane < a.c.dim
                     ? to_float(static_cast<const E*>(a.Q)[(row0 + r) * a.ldq + (h0 + q - r * p.gw) * a.c.dim + e * 32 + lane])
                     : 0.f;
        const int lead = __shfl_sync(~0u, tile.lead, r), len = __shfl_sync(~0u, tile.len, r);
        const int seq = __shfl_sync(~0u, tile.seq, r), first = __shfl_sync(~0u, tile.first, max(lead, 0));
        const long long t0 = (long long)(b0 - first) * kBlk, t1 = (long long)(b1 - first) * kBlk;
        if (len > 0)
          walk_tokens<E>(a, seq, int(max(t0, 0ll)), int(min(t1, (long long)len)), kv, x, m, l, o);
        const KvRowOut to = out(q, m, l, lane == 0);
#pragma unroll
        for (int e = 0; e < kLaneDims; ++e) {
          const float v[1] = {o[e]};
          if (e * 32 + lane < a.c.dim) put<E, 1>(to, e * 32 + lane, v);
        }
      }
    }
    if (opens) {
      // the workers up to the one with the item's last block
      const long long item_end = end + (tile.nb - b1);
      const int last = int((item_end * n + total - 1) / total) - 1;
      cut = make_int4(int(tile_id), unit, last - id + 1, 0);
    }
  }
  if (lane == 0) p.cuts[id] = cut;
  asm volatile("cp.async.wait_all;" ::: "memory");
  pdl_release();
}

// -------------------------------------------------------------------------- join ---
// Partial results of an item in order: warps take a query and some of its parts each, then add up.
constexpr int kJoinWarps = 16;

template <typename E>
__global__ void __launch_bounds__(kJoinWarps * 32) kv_join_kernel(const KvPass p) {
  __shared__ float part_o[kJoinWarps][kKvMaxDim];
  __shared__ float part_m[kJoinWarps], part_l[kJoinWarps];
  pdl_wait_and_release();
  const int id = blockIdx.x;
  const int4 cut = p.cuts[id];
  if (cut.z == 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, dim = p.a.c.dim;
  long long row0;
  const int n_rows = tile_rows(p, cut.x, row0);
  const int group = p.a.H / p.a.c.heads, kv = cut.y / p.gs, slice = (cut.y - kv * p.gs) * p.gw;
  const int gw = min(p.gw, group - slice), h0 = kv * group + slice, n_q = n_rows * gw;
  const int share = n_q >= kJoinWarps ? 1 : kJoinWarps / n_q;       // warps of a query
  const int stride = p.max_q * (dim + 2);
  for (int q0 = 0; q0 < n_q; q0 += kJoinWarps / share) {
    const int i = q0 + warp / share, sub = warp % share;
    const bool there = warp / share < kJoinWarps / share && i < n_q;
    const int r = there ? i / gw : 0, h = there ? i - r * gw : 0, q = r * p.gw + h;
    float m = kNegInf, l = 0.f, o[kLaneDims] = {};
    if (there)
#pragma unroll 4
      for (int k = sub; k < cut.z; k += share) {
        const float* base = p.parts + (long long)(k == 0 ? 2 * id + 1 : 2 * (id + k)) * stride;
        const float m2 = base[2 * q], l2 = base[2 * q + 1];
        const float* o2 = base + 2 * p.max_q + q * dim;
        float c, c2;
        join_state(m, l, c, c2, m2, l2);
#pragma unroll
        for (int e = 0; e < kLaneDims; ++e)
          if (e * 32 + lane < dim) o[e] = o[e] * c + o2[e * 32 + lane] * c2;
      }
    if (share > 1) {
#pragma unroll
      for (int e = 0; e < kLaneDims; ++e)
        if (e * 32 + lane < dim) part_o[warp][e * 32 + lane] = o[e];
      if (lane == 0) part_m[warp] = m, part_l[warp] = l;
      __syncthreads();
      if (there && sub == 0)
        for (int k = 1; k < share; ++k) {
          float c, c2;
          join_state(m, l, c, c2, part_m[warp + k], part_l[warp + k]);
#pragma unroll
          for (int e = 0; e < kLaneDims; ++e)
            if (e * 32 + lane < dim) o[e] = o[e] * c + part_o[warp + k][e * 32 + lane] * c2;
        }
      __syncthreads();
    }
    if (there && sub == 0) {
      const KvRowOut to = row_out(p, row0 + r, h0 + h, m, l, lane == 0);
#pragma unroll
      for (int e = 0; e < kLaneDims; ++e) {
        const float v[1] = {o[e]};
        if (e * 32 + lane < dim) put<E, 1>(to, e * 32 + lane, v);
      }
    }
  }
}

// ---------------------------------------------------------------------- launches ---
constexpr int kMostWorkers = 8 * kKvMostSms;

template <typename E>
cudaError_t run_join(const KvPass& p, cudaStream_t s) {
  return launch_pdl(kv_join_kernel<E>, dim3(p.workers), dim3(kJoinWarps * 32), 0, s, p);
}

template <typename Core>
cudaError_t run_pass(KvPass p, int sms, cudaStream_t s) {
  constexpr int kRing = Core::kWarps * (Core::kStages * 2 * kBlk * Core::kPacks * 16 + Core::kScratch);
  static_assert(kRing <= 220 * 1024, "the rings fit an SM");
  shape_pass(p, Core::kMaxQ, 32, kBlk);
  const int grid = std::min(sms, kKvMostSms);
  p.workers = grid * Core::kWarps;
  const cudaError_t e = cudaFuncSetAttribute(kv_blocks_kernel<Core>,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, kRing);
  if (e != cudaSuccess) return e;
  const cudaError_t f = launch_pdl(kv_blocks_kernel<Core>, dim3(grid), dim3(Core::kWarps * 32), kRing, s, p);
  return f != cudaSuccess ? f : run_join<typename Core::E>(p, s);
}

template <int kDim>
cudaError_t run_f32(const KvPass& p, int sms, cudaStream_t s) {
  const int group = p.a.H / p.a.c.heads;
  const long long q = std::min<long long>(p.part.per, p.a.N) * group;
  if (q <= 1) return run_pass<F32Core<kDim, 1>>(p, sms, s);
  if (q <= 4) return run_pass<F32Core<kDim, 4>>(p, sms, s);
  return run_pass<F32Core<kDim, 8>>(p, sms, s);
}

cudaError_t run_part(KvPass p, int sms, int* status, cudaStream_t s) {
  const int dim = p.a.c.dim;
  const long long queries = std::min<long long>(p.part.per, p.a.N) * (p.a.H / p.a.c.heads);
  if (p.a.c.dtype == 0 && dim <= 128 && queries > 16 && p.a.c.n_pages > 0 && p.a.scale >= 0.f) {
    const cudaError_t e = launch_kv_tc(p, sms, status, s);
    return e != cudaSuccess ? e : run_join<__nv_bfloat16>(p, s);
  }
  if (p.a.c.dtype == 0)
    return dim <= 32 ? run_pass<Bf16Core<32>>(p, sms, s) : dim <= 64 ? run_pass<Bf16Core<64>>(p, sms, s)
           : dim <= 128 ? run_pass<Bf16Core<128>>(p, sms, s) : run_pass<Bf16Core<256>>(p, sms, s);
  return dim <= 32 ? run_f32<32>(p, sms, s) : dim <= 64 ? run_f32<64>(p, sms, s)
         : dim <= 128 ? run_f32<128>(p, sms, s) : run_f32<256>(p, sms, s);
}

size_t up16(size_t x) { return (x + 15) / 16 * 16; }

struct Layout {
  size_t parts, cuts, pre_o, pre_ml, total;
};

Layout layout(long long N, int H, int dim, bool prefix) {
  Layout y;
  size_t at = 0;
  y.parts = at;
  at += up16(size_t(2 * kMostWorkers + 8) * 16 * (dim + 2) * sizeof(float));
  y.cuts = at;
  at += size_t(kMostWorkers) * sizeof(int4);
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

cudaError_t launch_kv_attention(const KvAttention& a, int sms, int* status, cudaStream_t s) {
  const Layout y = layout(a.N, a.H, a.c.dim, a.prefix_len != nullptr);
  char* ws = static_cast<char*>(a.ws);
  KvPass p{};
  p.a = a;
  p.parts = reinterpret_cast<float*>(ws + y.parts);
  p.cuts = reinterpret_cast<int4*>(ws + y.cuts);
  if (a.prefix_len != nullptr) {
    KvPass f = p;
    f.part = {a.prefix_seq, a.prefix_len, a.rows_per_prefix};
    f.put_o = reinterpret_cast<float*>(ws + y.pre_o);
    f.put_ml = reinterpret_cast<float*>(ws + y.pre_ml);
    const cudaError_t e = run_part(f, sms, status, s);
    if (e != cudaSuccess) return e;
    p.pre_o = f.put_o;
    p.pre_ml = f.put_ml;
  }
  p.part = {a.seq, a.len, a.rows_per_seq};
  return run_part(p, sms, status, s);
}

}  // namespace alr
