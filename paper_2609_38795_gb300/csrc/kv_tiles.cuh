// What the kernels of attention over the paged cache have in common: rows, tiles of rows, the even split
// of their tokens over workers, and where a row's result goes.
#pragma once

#include "kernels.h"
#include "row_reduce.cuh"

namespace alr {

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

// One pass over a part.  The rows go in tiles: groups of `per` consecutive rows (those that usually read
// the same sequence), each cut into `tg` tiles of `rows` rows.  A tile's tokens are those of its runs of
// rows with the same sequence, one run after the other, each in blocks of kBlk tokens; a tile of
// no tokens has one empty block, so that its rows are written.  An item is a tile and a unit, `gw` query
// heads of one key-value head (`gs` units a key-value head).
//   All items' blocks in order (tile, unit, block) are one line, and each worker takes an equal stretch
// of it, whatever the lengths are.  An item inside a stretch is finished by its worker; an item cut by a
// border leaves partial results, two a worker at most, which a second kernel joins in order.
struct KvPass {
  KvAttention a;
  KvPart part;
  int gw, gs, n_units;             // n_units = heads * gs
  int per, tg, rows;
  long long n_tiles;
  int step_pg, step_tok;           // kBlk tokens on: pages and tokens
  int workers;
  int max_q;                       // queries of an item, at most
  float* parts;                    // [2 * workers][max_q * (dim + 2)]: m and l of all queries, then o
  int4* cuts;                      // [workers]: (tile, unit, parts) of the item that a worker begins
                                   // and does not end; 0 parts: none
  float* put_o;                    // prefix pass: where results go, [N, H, dim] and [N, H, 2]
  float* put_ml;
  const float* pre_o;              // own pass after one: those results
  const float* pre_ml;
};

// Where a query's result goes, and the factors that turn its sums into it.
struct KvRowOut {
  float f, f_pre;          // of the sums, of the prefix's
  const float* pre;        // nullptr: none
  float* dst_f;            // partial results (fp32 sums) ...
  void* dst;               // ... or the final row
};

// Final or prefix destination of row r, head h with running maximum m (log2) and sum l.  `writer`: the
// one lane that writes the row's scalars.
ALR_DEV KvRowOut row_out(const KvPass& p, long long r, int h, float m, float l, bool writer) {
  KvRowOut o = {1.f, 0.f, nullptr, nullptr, nullptr};
  const int dim = p.a.c.dim;
  const long long i = r * p.a.H + h;
  if (p.put_o != nullptr) {
    o.dst_f = p.put_o + i * dim;
    if (writer) p.put_ml[2 * i] = m, p.put_ml[2 * i + 1] = l;
    return o;
  }
  float c = 1.f, c_pre = 0.f, top = m, sum = l;
  if (p.pre_o != nullptr) {
    const float m2 = p.pre_ml[2 * i], l2 = p.pre_ml[2 * i + 1];
    top = m > m2 ? m : m2;
    const float ref = top == kNegInf ? 0.f : top;
    c = m == ref ? 1.f : ex2(m - ref);
    c_pre = m2 == ref ? 1.f : ex2(m2 - ref);
    sum = l * c + l2 * c_pre;
    o.pre = p.pre_o + i * dim;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  o.f = c * inv;
  o.f_pre = c_pre * inv;
  const long long at = r * p.a.ldo + (long long)h * dim;
  o.dst = p.a.c.dtype == 0 ? static_cast<void*>(static_cast<__nv_bfloat16*>(p.a.out) + at)
                           : static_cast<void*>(static_cast<float*>(p.a.out) + at);
  if (writer && p.a.lse != nullptr) p.a.lse[i] = sum == 0.f ? kNegInf : top * kLn2 + logf(sum);
  return o;
}

// Partial results of query q in slot `slot`.
ALR_DEV KvRowOut part_out(const KvPass& p, long long slot, int q, float m, float l, bool writer) {
  float* base = p.parts + slot * p.max_q * (p.a.c.dim + 2);
  if (writer) base[2 * q] = m, base[2 * q + 1] = l;
  return {1.f, 0.f, nullptr, base + 2 * p.max_q + (long long)q * p.a.c.dim, nullptr};
}

// kW consecutive elements from d on.
template <typename E, int kW>
ALR_DEV void put(const KvRowOut& o, int d, const float (&v)[kW]) {
  struct alignas(kW * sizeof(float)) F { float e[kW]; };
  struct alignas(kW * sizeof(E)) T { E e[kW]; };
  F x;
#pragma unroll
  for (int i = 0; i < kW; ++i) x.e[i] = v[i] * o.f;
  if (o.dst_f != nullptr) {
    if constexpr (kW > 2) {      // partial rows begin at multiples of 8 bytes
#pragma unroll
      for (int i = 0; i < kW; i += 2) *reinterpret_cast<float2*>(o.dst_f + d + i) = {x.e[i], x.e[i + 1]};
    } else {
      *reinterpret_cast<F*>(o.dst_f + d) = x;
    }
    return;
  }
  if (o.pre != nullptr) {
#pragma unroll
    for (int i = 0; i < kW; ++i) x.e[i] = fmaf(o.pre[d + i], o.f_pre, x.e[i]);
  }
  T y;
#pragma unroll
  for (int i = 0; i < kW; ++i) y.e[i] = E(x.e[i]);
  *reinterpret_cast<T*>(static_cast<E*>(o.dst) + d) = y;
}

// Join two running results.
ALR_DEV void join_state(float& m, float& l, float& c, float& c2, float m2, float l2) {
  const float top = m > m2 ? m : m2, ref = top == kNegInf ? 0.f : top;
  c = m == ref ? 1.f : ex2(m - ref);
  c2 = m2 == ref ? 1.f : ex2(m2 - ref);
  l = l * c + l2 * c2;
  m = top;
}

}  // namespace alr
