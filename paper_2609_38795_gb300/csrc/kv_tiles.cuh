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

ALR_DEV int seen_len(const KvAttention& a, int seq, int len) {
  return seq < 0 || seq >= a.n_seq ? 0 : int(min((long long)max(len, 0), (long long)a.cols * a.c.page));
}

// One pass over a part.  The rows go in tiles: groups of `per` consecutive rows (those that usually read
// the same sequence), each cut into `tg` tiles of `rows` rows.  A tile's tokens are those of its runs of
// rows with the same sequence, one run after the other, each in blocks of kBlk tokens; a tile of
// no tokens has one empty block, so that its rows are written.  An item is a tile and a unit, `gw` query
// heads of one key-value head (`gs` units a key-value head).
//   All items in order (tile, unit), each with its blocks behind kItemCost places of no block (its queries,
// its results), are one line, and each worker takes an equal stretch of it, whatever the lengths
// are; a thread block's workers have consecutive stretches.  An item inside a
// stretch is finished by its worker; an item cut by a border leaves partial results, two a worker at
// most.  Its thread block joins those of its own workers in order, and a second kernel those of items
// that cross thread blocks, again two a block at most.
struct KvPass {
  KvAttention a;
  KvPart part;
  int gw, gs, n_units;             // n_units = heads * gs
  int per, tg, rows;
  int n_tiles;
  int step_pg, step_tok;           // kBlk tokens on: pages and tokens
  int block_workers;               // of a thread block, at most
  int stages;                      // blocks of a worker's ring
  bool one_each;                   // a thread block has one item, its line is the item's blocks
  int max_q;                       // queries of an item, at most
  float* parts;                    // [2 * workers][part_floats]: o of all queries, then m and l
  float* block_parts;              // [2 * blocks][part_floats]
  int4* cuts;                      // [blocks]: (tile, unit, parts) of the item that a block begins and
                                   // does not end; 0 parts: none
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

__host__ __device__ inline long long part_floats(int max_q, int dim) {
  return (long long)max_q * dim + (2 * max_q + 3) / 4 * 4;
}

// Partial results of query q in place `slot` of `parts`.
ALR_DEV KvRowOut part_out(const KvPass& p, float* parts, int slot, int q, float m, float l, bool writer) {
  float* base = parts + slot * part_floats(p.max_q, p.a.c.dim);
  float* ml = base + p.max_q * p.a.c.dim;
  if (writer) ml[2 * q] = m, ml[2 * q + 1] = l;
  return {1.f, 0.f, nullptr, base + q * p.a.c.dim, nullptr};
}

// kW consecutive elements from d on (a multiple of kW).  Workspaces are aligned to 16 bytes, no more.
template <typename E, int kW>
ALR_DEV void put(const KvRowOut& o, int d, const float (&v)[kW]) {
  struct alignas(kW < 4 ? kW * sizeof(float) : 16) F { float e[kW]; };
  struct alignas(kW * sizeof(E)) T { E e[kW]; };
  static_assert(kW * sizeof(E) <= 16, "a store of the result");
  if (o.dst_f != nullptr) {
    F x;
#pragma unroll
    for (int i = 0; i < kW; ++i) x.e[i] = v[i];
    *reinterpret_cast<F*>(o.dst_f + d) = x;
    return;
  }
  F pre = {};
  if (o.pre != nullptr) pre = *reinterpret_cast<const F*>(o.pre + d);
  T y;
#pragma unroll
  for (int i = 0; i < kW; ++i) y.e[i] = E(fmaf(pre.e[i], o.f_pre, v[i] * o.f));
  *reinterpret_cast<T*>(static_cast<E*>(o.dst) + d) = y;
}

// ---------------------------------------------------------------------- schedule ---
// First row and row count of a tile.
ALR_DEV int tile_rows(const KvPass& p, int tile, long long& row0) {
  const int g = tile / p.tg, i = tile - g * p.tg;
  row0 = (long long)g * p.per + (long long)i * p.rows;
  return int(min((long long)min(p.rows, p.per - i * p.rows), p.a.N - row0));
}

template <int kBlk>
ALR_DEV int blocks_of(int tokens) { return tokens / kBlk + (tokens % kBlk != 0); }

// Blocks of a tile, counted by one thread.
template <int kBlk>
ALR_DEV int tile_blocks(const KvPass& p, int tile) {
  long long row0;
  const int n = tile_rows(p, tile, row0);
  int nb = 0, cur = 0, most = 0;
  for (int i0 = 0; i0 < n; i0 += 8) {        // eight rows' loads at a time
    int s[8], len[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s[i] = i0 + i < n ? part_seq(p.part, row0 + i0 + i) : -1;
      len[i] = i0 + i < n ? p.part.len[row0 + i0 + i] : 0;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int k = seen_len(p.a, s[i], len[i]);
      if (k == 0) continue;
      if (most > 0 && s[i] != cur) {
        nb += blocks_of<kBlk>(most);
        most = 0;
      }
      cur = s[i];
      most = max(most, k);
    }
  }
  return max(nb + blocks_of<kBlk>(most), 1);
}

// A tile's runs, held by a warp: lane i has row i.
struct Tile {
  int seq, len;       // of the row
  int lead;           // first lane of the row's run (-1: before any)
  int first;          // of a run's first lane: its first block; INT_MAX elsewhere
  int most;           // ... and its longest row
  int nb;             // blocks (all lanes)
};

template <int kBlk>
ALR_DEV Tile load_tile(const KvPass& p, int tile) {
  const int lane = threadIdx.x & 31;
  long long row0;
  const int n = tile_rows(p, tile, row0);
  Tile t;
  t.seq = lane < n ? part_seq(p.part, row0 + lane) : -1;
  t.len = seen_len(p.a, t.seq, lane < n ? p.part.len[row0 + lane] : 0);
  const uint32_t some = __ballot_sync(~0u, t.len > 0), up_to = (2u << lane) - 1;
  const uint32_t before = some & (up_to >> 1);
  const int prev = __shfl_sync(~0u, t.seq, before != 0 ? 31 - __clz(before) : 0);
  const uint32_t leads = __ballot_sync(~0u, t.len > 0 && (before == 0 || prev != t.seq));
  t.lead = (leads & up_to) != 0 ? 31 - __clz(leads & up_to) : -1;
  t.most = t.len;
  for (int off = 1; off < p.rows; off <<= 1) {
    const int m = __shfl_down_sync(~0u, t.most, off), l = __shfl_down_sync(~0u, t.lead, off);
    if (lane + off < 32 && l == t.lead) t.most = max(t.most, m);
  }
  const bool lead = (leads >> lane & 1) != 0;
  const int nb = lead ? blocks_of<kBlk>(t.most) : 0, sum = warp_scan(nb);
  t.first = lead ? sum - nb : INT_MAX;
  t.nb = max(__shfl_sync(~0u, sum, 31), 1);
  return t;
}

// Position of a worker in the line of blocks.  The loads run ahead of the sums, so a worker has two.
template <int kBlk>
struct Cursor {
  Tile t;
  int tile, unit, b;
  int lead, seq, most, t0;      // the run's first lane, sequence, tokens; the block's first token
  int run_end;                  // first block of the next run

  ALR_DEV void enter() {
    const uint32_t m = __ballot_sync(~0u, t.first <= b);
    lead = m != 0 ? 31 - __clz(m) : -1;
    const int from = max(lead, 0);
    seq = __shfl_sync(~0u, t.seq, from);
    most = lead < 0 ? 0 : __shfl_sync(~0u, t.most, from);
    t0 = lead < 0 ? 0 : (b - __shfl_sync(~0u, t.first, from)) * kBlk;
    run_end = min(warp_min(t.first > b ? t.first : INT_MAX), t.nb);
  }
  ALR_DEV void start(const KvPass& p, int tile_, int unit_, int b_) {
    tile = tile_;
    unit = unit_;
    b = b_;
    t = load_tile<kBlk>(p, tile);
    enter();
  }
  // The rare part of a step, out of the loops' way (they run at the speed of their instructions' arrival).
  ALR_DEV static Cursor past_run(const KvPass& p, Cursor c) {
    if (c.b == c.t.nb) {
      c.b = 0;
      if (++c.unit == p.n_units) {
        c.unit = 0;
        ++c.tile;
        c.t = load_tile<kBlk>(p, c.tile);
      }
    }
    c.enter();
    return c;
  }
  // To the next block; whether it continues the run.
  ALR_DEV bool advance(const KvPass& p) {
    if (++b < run_end) {
      t0 += kBlk;
      return true;
    }
    *this = past_run(p, *this);
    return false;
  }
};

// a / b for a >= 0, b > 0: a 64-bit division costs half a microsecond, few are needed.
ALR_DEV long long quotient(long long a, long long b) {
  return ((a | b) >> 32) == 0 ? (long long)(uint32_t(a) / uint32_t(b)) : a / b;
}

// Blocks that an item costs beside its own.  Blocks of 16: decode of 64 x 0..32768 tokens by logarithm, whose
// short sequences come together, 153 us with 0, 138 with 2, 124 with 6 or 8; one of 64 x 0..1024 89, 69, 62.
// Blocks of 128: 128 blocks of 16 rows 278 us with 0, 257 with 2 or 4, 269 with 8.  (GPU time, cold.)
template <int kBlk>
constexpr int kItemCost = kBlk < 128 ? 6 : 3;

// The line: `n` workers (`per_block` consecutive ones of each thread block) have `each` places,
// the first `more` of them one more.
struct Line {
  long long each;
  int more, n, per_block;
  ALR_DEV long long start(int w) const { return w * each + min(w, more); }
  // Worker with the place before `end`.
  ALR_DEV int last_before(long long end) const {
    const long long i = end - 1 - more * (each + 1);
    return int(i < 0 ? quotient(end - 1, each + 1) : more + quotient(i, each));
  }
};

struct WorkerStart {
  long long block;             // number of its first block among all
  int tile, unit, b;
};

// Every thread block counts the places of all tiles, a thread some consecutive ones; a warp then finds the
// start of a worker among the warps' sums, its threads' and the tiles of the thread.  at[i]: start of the
// block's i-th worker, at[own workers]: of the next one.  Few blocks go to few workers of every thread block.
// sums: an entry a thread; buf: an entry a warp.
template <int kBlk>
ALR_DEV Line find_starts(const KvPass& p, WorkerStart* at, long long* sums, long long* buf) {
  using N = long long;
  const int tid = threadIdx.x, n_threads = blockDim.x, n_warps = n_threads / 32;
  const int lane = tid & 31, warp = tid >> 5;
  const int per = (p.n_tiles + n_threads - 1) / n_threads;
  const int a = int(min((long long)tid * per, (long long)p.n_tiles)), e = min(a + per, p.n_tiles);
  N own = 0;
  for (int i = a; i < e; ++i) own += tile_blocks<kBlk>(p, i) + kItemCost<kBlk>;
  own *= p.n_units;
  const N up = warp_scan(own);
  if (lane == 31) buf[warp] = up;
  __syncthreads();
  const N of_warps = warp_scan(lane < n_warps ? buf[lane] : N(0));
  const N total = __shfl_sync(~0u, of_warps, 31);
  const N before_warp = __shfl_sync(~0u, of_warps, max(warp - 1, 0));
  sums[tid] = (warp > 0 ? before_warp : N(0)) + up - own;
  Line line;
  const N items = N(p.n_tiles) * p.n_units, blocks = total - kItemCost<kBlk> * items;
  line.per_block = int(min(quotient(blocks + gridDim.x - 1, gridDim.x), (N)p.block_workers));
  line.n = int(min(N(line.per_block) * N(gridDim.x), blocks));
  const N each = quotient(total, line.n);
  line.each = each;
  line.more = int(total - each * line.n);
  __syncthreads();
  const int id0 = int(blockIdx.x) * line.per_block, n_own = min(line.per_block, line.n - id0);
  for (int k = warp; k <= n_own; k += n_warps) {
    if (id0 + k == line.n) {
      if (lane == 0) at[k] = {blocks, 0, 0, 0};
      continue;
    }
    const N pos = N(id0 + k) * each + min(id0 + k, line.more);
    // the last thread that begins at or before it
    const int w = __popc(__ballot_sync(~0u, lane < n_warps && sums[min(lane, n_warps - 1) * 32] <= pos)) - 1;
    const int n = w * 32 + __popc(__ballot_sync(~0u, sums[w * 32 + lane] <= pos));
    N rest = pos - sums[n - 1];
    const int tile_end = min(n * per, p.n_tiles);
    // rest is less than the thread's places (of lengths that do not change meanwhile)
    for (int tile = (n - 1) * per; tile < tile_end; tile += 32) {
      const int mine = tile + lane;
      const N len = mine < tile_end ? N(tile_blocks<kBlk>(p, mine) + kItemCost<kBlk>) * p.n_units : N(0);
      const N sum = per > 1 ? warp_scan(len) : len;
      const uint32_t past = __ballot_sync(~0u, sum > rest);
      if (past == 0) {
        rest -= __shfl_sync(~0u, sum, 31);
        continue;
      }
      const int k2 = __ffs(past) - 1;
      tile += k2;
      rest -= __shfl_sync(~0u, sum - len, k2);
      const N places = quotient(__shfl_sync(~0u, len, k2), p.n_units);
      const int unit = int(quotient(rest, places)), off = int(rest - unit * places);
      if (lane == 0)
        at[k] = {pos - kItemCost<kBlk> * (N(tile) * p.n_units + unit) - min(off, kItemCost<kBlk>), tile, unit,
                 max(off - kItemCost<kBlk>, 0)};
      break;
    }
  }
  __syncthreads();
  return line;
}

// The same where every thread block has one item.
template <int kBlk>
ALR_DEV Line find_item_starts(const KvPass& p, WorkerStart* at, long long* buf) {
  const int tile = blockIdx.x / p.n_units, unit = blockIdx.x - tile * p.n_units, tid = threadIdx.x;
  if (tid == 0) buf[0] = tile_blocks<kBlk>(p, tile);
  __syncthreads();
  const int nb = int(buf[0]);
  Line line;
  line.per_block = line.n = min(nb, p.block_workers);
  line.each = nb / line.n;
  line.more = nb - int(line.each) * line.n;
  if (tid <= line.n) {
    const int b = int(line.start(tid));
    at[tid] = {b, tile, unit, b};
  }
  __syncthreads();
  return line;
}

// ------------------------------------------------------------- a query by itself ---
// Weights of 0 times a value that is not finite are NaN, and such a value may lie in a token that a query
// does not see but another of its tile does, or whose score is -inf.  A query whose sums came out so is taken
// again over its tokens [t0, t1) of the item alone, by a warp, 32 tokens at a time: a score a lane, then the
// values of the tokens that count, four at a time by 8 lanes each.  Its result replaces the one in place: the
// final row or the prefix's, or with `parts` place `slot` there.
//   Rare, so short of registers first: 0.12 us a token and query for 64 bf16 elements, 0.21 for 128 (16 warps an
// SM, a million tokens a sequence; 0.83 and 1.08 by scores that a warp's lanes added up, token by token).
// kAhead: packs of values that a lane has on their way.
template <typename E, int kDim, int kAhead>
ALR_DEV void take_again(const KvPass& p, long long row, int h, int seq, int t0, int t1, float* parts,
                        int slot, int q) {
  constexpr int kPack = 16 / sizeof(E), kOwn = (kDim / kPack + 7) / 8;
  struct alignas(16) Pack { E e[kPack]; };
  const KvAttention& a = p.a;
  const int lane = threadIdx.x & 31, dim = a.c.dim, head = h / (a.H / a.c.heads);
  const int group = lane >> 3, first = (lane & 7) * kPack;           // of a token; the lane's packs
  const E* Q = static_cast<const E*>(a.Q) + row * a.ldq + (long long)h * dim;
  const E* K = static_cast<const E*>(a.c.K) + head * a.c.sh;
  const E* V = static_cast<const E*>(a.c.V) + head * a.c.sh;
  float m = kNegInf, l = 0.f, o[kOwn][kPack] = {};
  for (int b = t0; b < t1; b += min(32, t1 - b)) {
    int pg = -1;
    long long at = 0;
    if (lane < t1 - b) {
      const int t = b + lane, j = t / a.c.page;
      pg = a.table[(long long)seq * a.cols + j];
      at = pg * a.c.sp + (t - j * a.c.page) * a.c.st;
    }
    float x = kNegInf;
    if (pg >= 0 && pg < a.c.n_pages) {
      x = 0.f;
#pragma unroll 2 * kAhead
      for (int d = 0; d < dim; d += kPack) {
        const Pack k = *reinterpret_cast<const Pack*>(K + at + d), y = *reinterpret_cast<const Pack*>(Q + d);
#pragma unroll
        for (int e = 0; e < kPack; ++e) x = fmaf(to_float(y.e[e]), to_float(k.e[e]), x);
      }
      x = __fmul_rn(x, a.scale * kLog2e);
    }
    if (__any_sync(~0u, !(x < INFINITY))) {    // a score of NaN or +inf: so are all results
      l = NAN;
      break;
    }
    const uint32_t counts = __ballot_sync(~0u, x != kNegInf);
    if (counts == 0) continue;
    const float up = fmaxf(m, warp_max(x)), c = ex2(m - up), w = ex2(x - up);
    m = up;
    l = fmaf(l, c, w);
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
#pragma unroll
      for (int e = 0; e < kPack; ++e) o[i][e] *= c;
#pragma unroll kAhead
    for (int k0 = 0; k0 < 32; k0 += 4) {
      const int k = k0 + group;
      const E* v = V + __shfl_sync(~0u, at, k) + first;
      const float f = __shfl_sync(~0u, w, k);
#pragma unroll
      for (int i = 0; i < kOwn; ++i)
        if ((counts >> k & 1) && first + 8 * i * kPack < dim) {
          const Pack y = *reinterpret_cast<const Pack*>(v + 8 * i * kPack);
#pragma unroll
          for (int e = 0; e < kPack; ++e) o[i][e] = fmaf(f, to_float(y.e[e]), o[i][e]);
        }
    }
  }
  l = warp_reduce(l, AddOp());
  const KvRowOut to = parts == nullptr ? row_out(p, row, h, m, l, lane == 0)
                                       : part_out(p, parts, slot, q, m, l, lane == 0);
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
#pragma unroll
    for (int e = 0; e < kPack; ++e) {
      o[i][e] += __shfl_xor_sync(~0u, o[i][e], 8);
      o[i][e] += __shfl_xor_sync(~0u, o[i][e], 16);
    }
    if (group == 0 && first + 8 * i * kPack < dim) put<E, kPack>(to, first + 8 * i * kPack, o[i]);
  }
}

// Tokens [t0, t1) that row r of the tile sees of its run in blocks [b0, b1) (all lanes call it).
template <int kBlk>
ALR_DEV void row_tokens(const Tile& tile, int r, int b0, int b1, int& seq, int& t0, int& t1) {
  const int lead = __shfl_sync(~0u, tile.lead, r), len = __shfl_sync(~0u, tile.len, r);
  const int first = __shfl_sync(~0u, tile.first, max(lead, 0));
  seq = __shfl_sync(~0u, tile.seq, r);
  t0 = int(max((long long)(b0 - first) * kBlk, 0ll));
  t1 = len > 0 ? int(min((long long)(b1 - first) * kBlk, (long long)len)) : 0;
}

// A wait that runs out is recorded and passed over, as all waits after it: every role runs on to the end of
// its loop (on data that no one will use), so that no barrier is left half full.
ALR_DEV bool wait_longer(uint64_t* bar, uint32_t parity, volatile int* abort_word, int* status) {
  return !*abort_word && mbar_wait(bar, parity, AbortFlag{abort_word, status});
}
// For completion n (from 0) of `bar`; false: passed over.
ALR_DEV bool wait_on(uint64_t* bar, uint32_t n, const AbortFlag& ab) {
  return mbar_try_wait(bar, n & 1) || wait_longer(bar, n & 1, ab.smem, ab.status);
}

// Units, tiles and steps of a pass whose items have at most max_q queries in max_rows rows.
inline void shape_pass(KvPass& p, int max_q, int max_rows, int blk) {
  const int group = p.a.H / p.a.c.heads;
  const auto least = [](long long a, long long b) { return a < b ? a : b; };
  p.gs = (group + max_q - 1) / max_q;
  p.gw = (group + p.gs - 1) / p.gs;
  p.n_units = p.a.c.heads * p.gs;
  p.per = int(least(p.part.per, p.a.N));
  p.rows = int(least(least(max_q / p.gw, max_rows), p.per));
  p.tg = (p.per + p.rows - 1) / p.rows;
  p.rows = (p.per + p.tg - 1) / p.tg;
  p.n_tiles = int((p.a.N + p.per - 1) / p.per * p.tg);
  p.step_pg = blk / p.a.c.page;
  p.step_tok = blk % p.a.c.page;
  p.max_q = max_q;
}

constexpr int kKvMostSms = 160;

// kv_attention_tc.cu: a pass over tiles of up to 32 rows and 128 queries (bf16, dim <= 128, n_pages > 0,
// scale >= 0: references are maxima of the scores before they are scaled);
// p.part is set, the rest of the pass's shape is filled in.
cudaError_t launch_kv_tc(KvPass& p, const KvMaps& maps, int sms, int* status, cudaStream_t s);

}  // namespace alr
