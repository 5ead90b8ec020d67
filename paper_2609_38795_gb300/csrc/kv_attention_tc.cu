// Attention of many query rows that read the same tokens of the paged cache (a block of new tokens, rollouts
// with a shared prefix), on the 5th-generation tensor cores.
#include <algorithm>
#include <cfloat>

#include "launch.h"
#include "kv_tiles.cuh"

namespace alr {
namespace {

// Both products have the tokens or the elements of a value on their 128 rows and the queries on their
// columns, so that few queries waste nothing:
//   S^T [128 tokens, NQ] = K Q^T          (K tile and Q by rows of elements)
//   O^T [dim, NQ]       += V^T P^T        (V tile and P by rows of tokens, both read transposed)
// with S^T twice and O^T in tensor memory.  Bound by memory where the tokens are many (128 blocks of 16 rows over
// 1024 to 3000 tokens, 8 heads of 128, 4 queries a head: 245 us, 4.4 TB/s of the 1.08 GB read; a tile of 128
// tokens then takes 4200 cycles, of which a product's issue and wait 1000 each and a softmax 2200, one after
// the other on three roles), by the softmax where they are shared (6 prefixes of 2032 tokens, 128 rollouts each:
// 80 us).  A thread of the softmax has one token (a lane) and its
// group's queries (columns): no sum crosses lanes until the item ends, the weights leave as 16-byte packs
// into the shared-memory layout that the second product reads, and the running references are lagging
// ones, in shared memory: a tile whose scores stay below reference + kLag needs one vote of the threads.
//   Warps: groups of 4 for the softmax (each with its share of the queries), 4 copy (K and V
// tiles of 128 tokens, gathered by rows of their pages, in a ring), 1 issues products and 3 make its group
// whole.  A tile's softmax is a chain of waits more than work: four groups of 16 columns each take 297 us
// where two of 32 take 314, and loops that stay in the nearest instruction cache count for as much (issuing
// the products from rolled loops, 297 to 263; one place for all copies, 263 to 245).
//   A copy warp has 32 tokens of a tile.  Where a token's row is a row of one matrix over the whole cache
// and pages hold a multiple of 8 tokens, it fetches them by TMA in boxes of 8, 16 or 32 rows; the last
// tokens of a run and other layouts come by 16-byte copies, which an SM carries out at 24 bytes a cycle
// at most (all of it so: 300 us cold where boxes take 257; by tile::gather4, which would serve any page, it
// took 644 where these copies took 353).
constexpr int kBlk = 128;
constexpr int kCopyWarps = 4;
constexpr int kInfo = 8;           // tiles whose masks and flags are kept
constexpr float kLag = 8.f;        // log2: weights of up to 2^8 relative to the reference
constexpr float kNoRef = -FLT_MAX;

template <int kNQ_, int kChunks_>
struct Cfg {
  static constexpr int kNQ = kNQ_, kChunks = kChunks_;     // queries; 64-element chunks of a row
  static constexpr int kTile = kChunks * kBlk * 128;       // bytes of a K or V tile
  static constexpr int kQBytes = kChunks * kNQ * 128;
  static constexpr int kPBytes = (kNQ / 64) * kBlk * 128;
  static constexpr int kQBufs = 2, kPBufs = kNQ == 128 && kChunks == 2 ? 1 : 2;
  static constexpr int kSlots = kChunks == 1 ? 8 : kNQ == 128 ? 4 : 5;
  static constexpr int kGroups = 4;                        // of 4 softmax warps
  static constexpr int kOwn = kNQ / kGroups;               // queries of a group ...
  static constexpr int kW = 16;                            // ... and columns at a time (tmem_ld16)
  static constexpr int kParts = kOwn / kW;
  static constexpr int kSoftWarps = 4 * kGroups, kCopyWarp = kSoftWarps, kMmaWarp = kCopyWarp + kCopyWarps;
  static constexpr int kWarps = kMmaWarp + 4, kThreads = kWarps * 32;
  // Registers: 80 a thread at the launch; groups with 32 columns' sums take some from the other warps.
  static constexpr int kSoftRegs = kNQ == 128 ? 88 : 0, kOtherRegs = kNQ == 128 ? 64 : 0;
  static_assert(kGroups * kSoftRegs + 2 * kOtherRegs <= (kGroups + 2) * 80, "the launch's registers");
  static constexpr int kCols = kNQ == 128 ? 512 : 256;     // tensor memory: S^T, S^T, O^T
  static constexpr size_t kBig = size_t(kSlots) * kTile + kQBufs * kQBytes + kPBufs * kPBytes;
};

struct alignas(16) KvMisc {
  uint64_t full[8], empty[8], q_empty[2], s_full[2], s_empty[2], p_full[2], pv_done[2], drain;
  uint32_t there[kInfo][kCopyWarps];      // tokens of a tile whose page exists
  uint32_t info[kInfo];                   // 1: first of its item here, 2: last
  uint32_t tmem;
  int abort_word;
  int odd;                                // whether some result was not finite
  WorkerStart start[2];
  Line line;                              // needed again at the end alone
  long long buf[24];
};

template <class C>
struct KvSmem {
  KvMisc m;
  float top[C::kSoftWarps][C::kW];        // a slow tile's maxima
  float ref[C::kNQ];                      // references (scores)
  int vis[C::kNQ];                        // tokens of the run that a query sees
};
static_assert(sizeof(KvMisc) % 16 == 0, "what follows is read as packs of 16 bytes");

// At an item's end: sums and destinations of all queries, and each group's place to turn kW queries' rows.
template <class C>
constexpr int end_bytes() { return C::kSoftWarps * C::kOwn * 4 + C::kNQ * int(sizeof(KvRowOut)); }
template <class C>
constexpr int stage_bytes() { return C::kW * C::kChunks * 128; }

template <class C>
constexpr size_t smem_bytes() { return C::kBig + sizeof(KvSmem<C>); }

ALR_DEV void cp_async16_or_zero(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0)
               : "memory");
}
// Arrive on `bar` once all copies this thread issued so far have landed.
ALR_DEV void cp_async_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
ALR_DEV bool any_of(int id, int threads, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r) : "r"(x ? 1u : 0u), "r"(id), "r"(threads) : "memory");
  return r != 0;
}
ALR_DEV void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
                 "=r"(r[7])
               : "r"(taddr));
}
ALR_DEV void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
      "%14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
ALR_DEV void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(taddr)
               : "memory");
}
ALR_DEV void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

ALR_DEV uint32_t bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// More bytes to come for `bar` in its present phase.
ALR_DEV void mbar_expect_tx(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes)
               : "memory");
}

// A place of the ring; tiles are copied and used in the order K0 K1 V0 K2 V1 ... K(n-1) V(n-2) V(n-1).
template <int kSlots>
struct Place {
  int slot = 0;
  uint32_t round = 0;
  ALR_DEV void next() {
    if (++slot == kSlots) slot = 0, ++round;
  }
};

// The slow tile of a softmax group: the references of kW columns move to the maxima with this tile, the
// products so far (if any) are scaled.  Lane k returns the factor of column k (mod kW).  pos: the thread's token,
// INT_MAX if its page does not exist.
template <int kW>
__device__ __noinline__ float move_refs(uint32_t s_at, uint32_t o_at, float c, float* ref, const int* vis,
                                        float (*top)[kW], int bar, int pos, bool scale_o) {
  const int lane = threadIdx.x % kW, wq = threadIdx.x >> 5 & 3;
  float most = kNegInf;
#pragma unroll 1
  for (int k0 = 0; k0 < kW; k0 += 8) {
    uint32_t s[8];
    tmem_ld8(s_at + k0, s);
    tmem_ld_wait();
    reg_fence(s);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float m = warp_max(pos < vis[k0 + k] ? __uint_as_float(s[k]) : kNegInf);
      if (lane == k0 + k) most = m;
    }
  }
  top[wq][lane] = most;
  named_bar_sync(bar, 128);
  const float old = ref[lane];
  float up = old;
  for (int k = 0; k < 4; ++k) up = fmaxf(up, top[k][lane]);
  const float f = old == up ? 1.f : ex2((old - up) * c);
  named_bar_sync(bar, 128);
  if (wq == 0) ref[lane] = up;
  if (scale_o) {
#pragma unroll 1
    for (int k0 = 0; k0 < kW; k0 += 8) {
      uint32_t s[8];
      tmem_ld8(o_at + k0, s);
      tmem_ld_wait();
      reg_fence(s);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        s[k] = __float_as_uint(__uint_as_float(s[k]) * __shfl_sync(~0u, f, k0 + k));
      tmem_st8(o_at + k0, s);
    }
    tmem_st_wait();
  }
  named_bar_sync(bar, 128);
  return f;
}

// The results of worker `id`'s stretch that are not finite, each taken again by one of n_warps warps.  They are
// found where they were left: a list of them would have no bound.
template <typename E, int kDim>
__device__ __noinline__ void take_odd_again(const KvPass& p, const WorkerStart& from, int count, int id, int warp,
                                            int n_warps) {
  const int lane = threadIdx.x & 31, dim = p.a.c.dim, group = p.a.H / p.a.c.heads;
  int tile_id = from.tile, unit = from.unit, b0 = from.b;
  while (count > 0) {
    const Tile tile = load_tile<kBlk>(p, tile_id);
    long long row0;
    const int n_rows = max(tile_rows(p, tile_id, row0), 0), b1 = min(tile.nb, b0 + count);
    const int kv = unit / p.gs, slice = (unit - kv * p.gs) * p.gw, gw = min(p.gw, group - slice);
    const bool whole = b0 == 0 && b1 == tile.nb, opens = b0 == 0 && b1 < tile.nb;
    const int part = 2 * id + (opens ? 1 : 0);
    for (int q = warp; q < n_rows * p.gw; q += n_warps) {
      const int r = q / p.gw, h = kv * group + slice + q - r * p.gw;
      if (q - r * p.gw >= gw) continue;
      const float* sums = whole ? p.put_o + ((row0 + r) * p.a.H + h) * dim
                                : p.block_parts + part * part_floats(p.max_q, dim) + q * dim;
      const E* row = static_cast<const E*>(p.a.out) + (row0 + r) * p.a.ldo + (long long)h * dim;
      const bool final_row = whole && p.put_o == nullptr;
      float odd = 0.f;
      for (int d = lane; d < dim; d += 32) odd = fmaf(0.f, final_row ? to_float(row[d]) : sums[d], odd);
      if (!__any_sync(~0u, !(odd == 0.f))) continue;
      int seq, t0, t1;
      row_tokens<kBlk>(tile, r, b0, b1, seq, t0, t1);
      take_again<E, kDim, 2>(p, row0 + r, h, seq, t0, t1, whole ? nullptr : p.block_parts, part, q);
    }
    count -= b1 - b0;
    b0 = 0;
    if (++unit == p.n_units) unit = 0, ++tile_id;
  }
}

template <class C>
__global__ void __launch_bounds__(C::kThreads, 1)
    kv_tc_kernel(const __grid_constant__ KvMaps maps, const __grid_constant__ KvPass p, int* status) {
  using E = __nv_bfloat16;
  constexpr int kNQ = C::kNQ, kSlots = C::kSlots, kThreads = C::kThreads;
  constexpr int kSoftWarps = C::kSoftWarps, kCopyWarp = C::kCopyWarp, kMmaWarp = C::kMmaWarp;
  extern __shared__ __align__(1024) uint8_t tc_smem[];
  uint8_t* ring = tc_smem;
  uint8_t* qs = ring + kSlots * C::kTile;
  uint8_t* ps = qs + C::kQBufs * C::kQBytes;
  KvSmem<C>& sm = *reinterpret_cast<KvSmem<C>*>(ps + C::kPBufs * C::kPBytes);
  KvMisc& mi = sm.m;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const KvAttention& a = p.a;
  const int dim = a.c.dim;
  const AbortFlag ab{&mi.abort_word, status};
  if (threadIdx.x == 0) {
    for (int i = 0; i < kSlots; ++i) {
      // every copying thread's copies, and its warp's flags; one that never comes: withheld
      mbar_init(&mi.full[i], kCopyWarps * 33 + (i == 0 && p.a.withhold_first_stage ? 1 : 0));
      mbar_init(&mi.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&mi.q_empty[i], 1);
      mbar_init(&mi.s_full[i], 1);
      mbar_init(&mi.s_empty[i], kSoftWarps);
      mbar_init(&mi.p_full[i], kSoftWarps);
      mbar_init(&mi.pv_done[i], 1);
    }
    mbar_init(&mi.drain, 1);
    mi.abort_word = 0;
    mi.odd = 0;
    fence_mbar_init();
  }
  if (warp == kMmaWarp) {
    tmem_alloc(&mi.tmem, C::kCols);
    tmem_relinquish();
  }
  tc_fence_before();
  pdl_wait();
  const Line line = find_starts<kBlk>(p, mi.start, reinterpret_cast<long long*>(ring), mi.buf);   // barriers within
  tc_fence_after();
  if (dim % 16 != 0) {                       // what lies past a row's end is never copied: zeros
    uint4* z = reinterpret_cast<uint4*>(ring);
    for (int i = threadIdx.x; i < (kSlots * C::kTile + C::kQBufs * C::kQBytes) / 16; i += kThreads)
      z[i] = make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async_smem();                  // the copies come after this and the sums of the starts
  __syncthreads();
  const uint32_t tmem = mi.tmem;
  const int id = blockIdx.x;                 // the block's one worker
  const int count = id < line.n ? int(mi.start[1].block - mi.start[0].block) : 0;
  if (threadIdx.x == 0) mi.line = line;
  if (threadIdx.x == 0 && count == 0) p.cuts[id] = make_int4(0, 0, 0, 0);

  if (warp >= kCopyWarp && warp < kMmaWarp) {
    // ---- copies
    if constexpr (C::kOtherRegs > 0) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kOtherRegs));
    const int w = warp - kCopyWarp;
    constexpr int kRowsAt = 4 / C::kChunks, kPer = 32 / kRowsAt;     // rows of one copy instruction
    const int pack = lane & (8 * C::kChunks - 1), sub = lane / (8 * C::kChunks);
    const bool has_pack = pack * 8 < dim;
    // place of (row r of the tile, this pack): the low bits of r swizzle the packs of 128 bytes
    const uint32_t ring_at = smem_u32(ring), q_at = smem_u32(qs);
    const auto place = [&](int r, int rows) {
      return uint32_t((pack >> 3) * rows * 128 + r * 128 + (((pack & 7) ^ (r & 7)) << 4));
    };
    Cursor<kBlk> in{};
    // What a tile's copies need.  The table is read a tile ahead: a page's number takes as long to come
    // as its rows.
    struct Next {
      int pg, off, unit, tile;
      bool first, last, whole;               // whole: all of the warp's tokens are the run's
    } next = {-1, 0, 0, 0, true, true, false};
    int j = 0, off = 0;
    const auto look_up = [&](bool runs_on, int i) {
      if (runs_on) {
        j += p.step_pg;
        off += p.step_tok;
        if (off >= a.c.page) off -= a.c.page, ++j;
      } else {
        const int tok = in.t0 + w * 32 + lane;
        j = tok / a.c.page;
        off = tok - j * a.c.page;
      }
      next.pg = in.t0 + w * 32 + lane < in.most ? a.table[(long long)in.seq * a.cols + j] : -1;
      next.off = off;
      next.whole = in.most - in.t0 >= w * 32 + 32;
      next.unit = in.unit;
      next.tile = in.tile;
      next.first = i == 0 || in.b == 0;
      next.last = i + 1 == count || in.b + 1 == in.t.nb;
    };
    if (count > 0) {
      in.start(p, mi.start[0].tile, mi.start[0].unit, mi.start[0].b);
      look_up(false, 0);
    }
    Place<kSlots> to;
    // box: first matrix row of the lane's box of the warp's tokens, -1: copies of 16 bytes
    const int n_boxes = maps.box_rows > 0 ? 32 / maps.box_rows : 0, n_chunks = (dim + 63) / 64;
    bool stop = false;
    const auto copy = [&](const void* cache, const CUtensorMap* map, int kv, long long row, uint32_t all, int box) {
      // Without its place empty nothing more is copied: copies of two rounds would count for one phase of the
      // place's barrier.
      if (to.round > 0 && !wait_on(&mi.empty[to.slot], to.round - 1, ab)) stop = true;
      if (__any_sync(~0u, stop)) {
        stop = true;
        return;
      }
      if (box >= 0) {
        if (lane < n_boxes) {
          mbar_expect_tx(&mi.full[to.slot], n_chunks * maps.box_rows * 128);
          for (int c = 0; c < n_chunks; ++c)
            tma_load_2d(ring + to.slot * C::kTile + c * (kBlk * 128) + (w * 32 + lane * maps.box_rows) * 128, map,
                        &mi.full[to.slot], kv * maps.head_cols + c * 64, box);
        }
        cp_async_arrive(&mi.full[to.slot]);
        __syncwarp();
        if (lane == 0) mbar_arrive(&mi.full[to.slot]);
        to.next();
        return;
      }
      const E* base = static_cast<const E*>(cache) + kv * a.c.sh + pack * 8;
      const uint32_t dst = ring_at + to.slot * C::kTile;
#pragma unroll 4
      for (int i = 0; i < kPer; ++i) {
        const int r = i * kRowsAt + sub;
        const long long from = __shfl_sync(~0u, row, r);
        if (has_pack) cp_async16_or_zero(dst + place(w * 32 + r, kBlk), base + from, all >> r & 1);
      }
      cp_async_arrive(&mi.full[to.slot]);
      __syncwarp();
      if (lane == 0) mbar_arrive(&mi.full[to.slot]);
      to.next();
    };
    long long row_v = 0;
    uint32_t all_v = 0;
    int kv_v = 0, item = -1, box_v = -1;
#pragma unroll 1
    for (int i = 0; i <= count && count > 0 && !stop; ++i) {
      const Next cur = next;
      if (i + 1 < count) {
        const bool on = in.advance(p);
        look_up(on, i + 1);
      }
      long long row = 0;
      uint32_t all = 0;
      int kv = 0, box = -1;
      if (i < count) {
        const bool there = cur.pg >= 0 && cur.pg < a.c.n_pages;
        all = __ballot_sync(~0u, there);
        row = there ? cur.pg * a.c.sp + cur.off * a.c.st : 0;
        kv = cur.unit / p.gs;
        if (n_boxes > 0 && cur.whole) {
          const int from = (lane * maps.box_rows) & 31;
          const int pg = __shfl_sync(~0u, there ? cur.pg : -1, from), off = __shfl_sync(~0u, cur.off, from);
          box = pg >= 0 ? pg * maps.page_rows + off + kv * maps.head_rows : maps.n_rows;   // past the end: zeros
        }
        // flags and masks of tile i: read after its keys have landed; tile i - kInfo is long done with
        // (its values' slot has been refilled since)
        if (lane == 0) {
          mi.there[i % kInfo][w] = all;
          if (w == 0) mi.info[i % kInfo] = (cur.first ? 1u : 0u) | (cur.last ? 2u : 0u);
        }
        if (cur.first) {
          ++item;
          if (item >= 2) wait_on(&mi.q_empty[item & 1], (item >> 1) - 1, ab);
          long long row0;
          const int n_rows = max(tile_rows(p, cur.tile, row0), 0);
          const int group_q = a.H / a.c.heads, slice = (cur.unit - kv * p.gs) * p.gw;
          const int gw = min(p.gw, group_q - slice), h0 = kv * group_q + slice;
          const uint32_t dst = q_at + (item & 1) * C::kQBytes;
          for (int q = w * kRowsAt + sub; q < kNQ; q += kCopyWarps * kRowsAt) {
            const int r = q / p.gw, h = q - r * p.gw;
            const bool ok = r < n_rows && h < gw;
            const E* src = static_cast<const E*>(a.Q) + (ok ? (row0 + r) * a.ldq + (long long)(h0 + h) * dim : 0);
            if (has_pack) cp_async16_or_zero(dst + place(q, kNQ), src + pack * 8, ok);
          }
        }
      }
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {          // keys of tile i, values of the tile before
        if (h == 0 ? i == count : i == 0 || stop) continue;
        copy(h == 0 ? a.c.K : a.c.V, h == 0 ? &maps.k : &maps.v, h == 0 ? kv : kv_v, h == 0 ? row : row_v,
             h == 0 ? all : all_v, h == 0 ? box : box_v);
      }
      box_v = box;
      row_v = row;
      all_v = all;
      kv_v = kv;
    }
    if (*ab.smem)                            // no copy outlives the block
      for (int k = 0; k < kSlots; ++k) {
        const int round = int(to.round) - (k < to.slot ? 0 : 1);
        if (round >= 0) mbar_wait_drain(&mi.full[k], round & 1);
      }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp >= kMmaWarp) {
    // ---- products
    if constexpr (C::kOtherRegs > 0) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kOtherRegs));
    if (warp == kMmaWarp && lane == 0 && count > 0) {
      constexpr uint32_t i_s = idesc_make(false, 128, kNQ, false, false);
      constexpr uint32_t i_o = idesc_make(false, 128, kNQ, true, true);
      const int n_k = (dim + 15) / 16;
      // Descriptors of the first places; others are so many 16 bytes further.  One thread issues, and every
      // instruction between two products is time: unrolled loops, whose instructions come from beyond the
      // nearest cache, took 110 cycles a product.
      const uint64_t k_desc = sdesc_sw128(smem_u32(ring), 16, 1024), q_desc = sdesc_sw128(smem_u32(qs), 16, 1024);
      const uint64_t v_desc = sdesc_sw128(smem_u32(ring), kBlk * 128, 1024);
      const uint64_t p_desc = sdesc_sw128(smem_u32(ps), kBlk * 128, 1024);
      int item = -1;
      uint32_t prev = 0;
      bool gone = false;                     // a place was not filled in time: none is called empty any more
      Place<kSlots> from;
      // The proxy fences here, after the waits, order the copies' and the softmax's writes to shared
      // memory before the products' reads (a fence in every writing thread cost 360 cycles a tile).
      const auto values = [&](int i, uint32_t info) {
        const int pb = C::kPBufs == 2 ? i & 1 : 0;
        if (!wait_on(&mi.full[from.slot], from.round, ab)) gone = true;
        wait_on(&mi.p_full[pb], C::kPBufs == 2 ? i >> 1 : i, ab);
        fence_proxy_async_smem();
        tc_fence_after();
        // dim <= 64: rows 64 to 127 of the result come from whatever lies behind the tile, unused
        uint64_t va = v_desc + from.slot * (C::kTile >> 4), pa = p_desc + pb * (C::kPBytes >> 4);
        uint32_t add = !(info & 1);
#pragma unroll 1
        for (int k = 0; k < kBlk / 16; ++k, va += 2048 >> 4, pa += 2048 >> 4, add = 1)
          mma_issue<false>(tmem + 2 * kNQ, va, pa, i_o, add);
        if (!gone) mma_commit(&mi.empty[from.slot]);
        mma_commit(&mi.pv_done[pb]);
        from.next();
      };
#pragma unroll 1
      for (int i = 0; i <= count; ++i) {
        uint32_t info = 0;
        if (i < count) {
          const int sb = i & 1;
          if (!wait_on(&mi.full[from.slot], from.round, ab)) gone = true;
          info = mi.info[i % kInfo];
          if (info & 1) ++item;
          if (i >= 2) wait_on(&mi.s_empty[sb], (i >> 1) - 1, ab);
          fence_proxy_async_smem();
          tc_fence_after();
          uint64_t ka = k_desc + from.slot * (C::kTile >> 4), qa = q_desc + (item & 1) * (C::kQBytes >> 4);
#pragma unroll 1
          for (int k = 0; k < n_k; ++k) {
            mma_issue<false>(tmem + sb * kNQ, ka, qa, i_s, k);
            // 32 bytes on, or to the next chunk of 64 elements
            ka += (k & 3) == 3 ? (kBlk * 128 - 96) >> 4 : 32 >> 4;
            qa += (k & 3) == 3 ? (kNQ * 128 - 96) >> 4 : 32 >> 4;
          }
          if (!gone) mma_commit(&mi.empty[from.slot]);
          mma_commit(&mi.s_full[sb]);
          if (info & 2) mma_commit(&mi.q_empty[item & 1]);
          from.next();
        }
        if (i > 0) values(i - 1, prev);
        prev = info;
      }
      mma_commit(&mi.drain);                 // nothing is in flight when the memory is given back
      mbar_wait_drain(&mi.drain, 0);
    }
    __syncwarp();
  } else {
    // ---- softmax
    if constexpr (C::kSoftRegs > 0) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kSoftRegs));
    constexpr int kOwn = C::kOwn, kW = C::kW, kParts = C::kParts, kAllBar = 5, kAll = kSoftWarps * 32;
    const int wg = warp >> 2, wq = warp & 3, bar = 1 + wg, tid = threadIdx.x & 127;
    const uint32_t lanes = tmem + (uint32_t(wq * 32) << 16);
    const int tok = tid, q0 = wg * kOwn;
    const float c = a.scale * kLog2e;
    const uint64_t c2 = f2_pack(c, c);
    float l[kOwn];
    Cursor<kBlk> at;
    if (count > 0) at.start(p, mi.start[0].tile, mi.start[0].unit, mi.start[0].b);
    float (*lsum)[kOwn] = reinterpret_cast<float (*)[kOwn]>(ps);               // at an item's end
    KvRowOut* outs = reinterpret_cast<KvRowOut*>(ps + kSoftWarps * kOwn * sizeof(float));
    constexpr int kEndBytes = end_bytes<C>(), kStageBytes = stage_bytes<C>();
    int4 cut = make_int4(0, 0, 0, 0);
    int i = 0;
    while (i < count) {
      long long row0;
      const int n_rows = max(tile_rows(p, at.tile, row0), 0);
      const int group_q = a.H / a.c.heads, kv = at.unit / p.gs, slice = (at.unit - kv * p.gs) * p.gw;
      const int gw = min(p.gw, group_q - slice), h0 = kv * group_q + slice, n_q = n_rows * p.gw;
      const Tile tile = at.t;
      const int tile_id = at.tile, unit = at.unit, b0 = at.b, b1 = min(tile.nb, b0 + (count - i));
      const int i0 = i;
      if (tid < kOwn) sm.ref[q0 + tid] = kNoRef;
#pragma unroll
      for (int k = 0; k < kOwn; ++k) l[k] = 0.f;
      int run = -2, least = 0;
      for (int b = b0; b < b1; ++b, ++i) {
        if (at.lead != run) {
          // tokens that the queries see of the run
          run = at.lead;
          const int see = run >= 0 && tile.lead == run ? tile.len : 0;
          least = warp_min(lane < n_rows ? see : INT_MAX);
          named_bar_sync(bar, 128);
          if (wq == 0)
            for (int k = 0; k < kOwn; k += 32) {
              const int q = q0 + k + lane, v = __shfl_sync(~0u, see, (q / p.gw) & 31);
              if (k + lane < kOwn) sm.vis[q] = q < n_q ? v : INT_MAX;
            }
          named_bar_sync(bar, 128);
        }
        const int sb = i & 1, pb = C::kPBufs == 2 ? i & 1 : 0;
        wait_on(&mi.s_full[sb], i >> 1, ab);
        tc_fence_after();
        const uint32_t* there = mi.there[i % kInfo];
        const int pos = there[wq] >> lane & 1 ? at.t0 + tok : INT_MAX;
        const bool plain = least - at.t0 >= kBlk && (there[0] & there[1] & there[2] & there[3]) == ~0u;
        const uint32_t s_at = lanes + sb * kNQ + q0, o_at = lanes + 2 * kNQ + q0;
        uint8_t* prow = ps + pb * C::kPBytes + tok * 128;
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
          float y[kW];
          // Exponents are differences of scores, times c (the fma s c - ref c would leave the rounding of
          // ref c, which is more than 2^8 from |ref c| = 2^32 on): after a move none is above 0.
          for (bool moved = false;; moved = true) {
            uint32_t s[16];
            tmem_ld16(s_at + part * kW, s);
            const float* ref = sm.ref + q0 + part * kW;
            float t = kNegInf;
            tmem_ld_wait();
            reg_fence(s);
#pragma unroll
            for (int k = 0; k < kW; k += 4) {
              const float4 r = *reinterpret_cast<const float4*>(ref + k);
              f2_unpack(f2_mul(f2_sub(f2_pack(__uint_as_float(s[k]), __uint_as_float(s[k + 1])),
                                      f2_pack(r.x, r.y)), c2), y[k], y[k + 1]);
              f2_unpack(f2_mul(f2_sub(f2_pack(__uint_as_float(s[k + 2]), __uint_as_float(s[k + 3])),
                                      f2_pack(r.z, r.w)), c2), y[k + 2], y[k + 3]);
            }
            if (!plain) {
              const int* vis = sm.vis + q0 + part * kW;
#pragma unroll
              for (int k = 0; k < kW; k += 4) {
                const int4 r = *reinterpret_cast<const int4*>(vis + k);
                y[k] = pos < r.x ? y[k] : kNegInf;
                y[k + 1] = pos < r.y ? y[k + 1] : kNegInf;
                y[k + 2] = pos < r.z ? y[k + 2] : kNegInf;
                y[k + 3] = pos < r.w ? y[k + 3] : kNegInf;
              }
            }
#pragma unroll
            for (int k = 0; k < kW; k += 2) t = max3(t, y[k], y[k + 1]);
            if (moved || !any_of(bar, 128, t > kLag)) break;
            if (i > i0) {
              wait_on(&mi.pv_done[C::kPBufs == 2 ? (i - 1) & 1 : 0], C::kPBufs == 2 ? (i - 1) >> 1 : i - 1, ab);
              tc_fence_after();
            }
            const float f = move_refs<kW>(s_at + part * kW, o_at + part * kW, c, sm.ref + q0 + part * kW,
                                      sm.vis + q0 + part * kW, sm.top + wg * 4, bar, pos, i > i0);
#pragma unroll
            for (int k = 0; k < kW; ++k) l[part * kW + k] *= __shfl_sync(~0u, f, k);
          }
          // this buffer's last product
          if (part == 0 && i >= C::kPBufs)
            wait_on(&mi.pv_done[pb], C::kPBufs == 2 ? (i >> 1) - 1 : i - 1, ab);
#pragma unroll
          for (int k = 0; k < kW; k += 8) {
            uint32_t x[4];
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
              const float u = ex2(y[k + e]), v = ex2(y[k + e + 1]);
              l[part * kW + k + e] += u;
              l[part * kW + k + e + 1] += v;
              x[e / 2] = bf16x2(u, v);   // the product's only operand type: off by 2^-8, l is not
            }
            const int q = q0 + part * kW + k;
            *reinterpret_cast<uint4*>(prow + (q >> 6) * (kBlk * 128) + ((((q & 63) >> 3) ^ (tok & 7)) << 4)) =
                make_uint4(x[0], x[1], x[2], x[3]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&mi.s_empty[sb]);
          mbar_arrive(&mi.p_full[pb]);
        }
        if (i + 1 < count) at.advance(p);
      }
      // ---- the item's results
      wait_on(&mi.pv_done[C::kPBufs == 2 ? (i - 1) & 1 : 0], C::kPBufs == 2 ? (i - 1) >> 1 : i - 1, ab);
      tc_fence_after();
      named_bar_sync(kAllBar, kAll);                // all groups are past their last weights
      // sums over the warp's tokens: lane k ends with column k's
#pragma unroll
      for (int part = 0; part < kParts; ++part) {
#pragma unroll
        for (int off = kW / 2; off > 0; off >>= 1) {
          const bool upper = (lane & off) != 0;
#pragma unroll
          for (int k = 0; k < off; ++k) {
            float& lo = l[part * kW + k];
            const float hi = l[part * kW + k + off];
            const float give = upper ? lo : hi, keep = upper ? hi : lo;
            lo = keep + __shfl_xor_sync(~0u, give, off);
          }
        }
        float sum = l[part * kW];
        sum += __shfl_xor_sync(~0u, sum, 16);
        if (lane < kW) lsum[warp][part * kW + lane] = sum;
      }
      named_bar_sync(bar, 128);
      const bool whole = b0 == 0 && b1 == tile.nb, opens = b0 == 0 && b1 < tile.nb;
      const int part_id = 2 * id + (opens ? 1 : 0);
      const auto out = [&](int q, int r, float m, float s, bool writer) {
        return whole ? row_out(p, row0 + r, h0 + q - r * p.gw, m, s, writer)
                     : part_out(p, p.block_parts, part_id, q, m, s, writer);
      };
      if (tid < kOwn) {
        const int q = q0 + tid, r = q / p.gw;
        float s = 0.f;
        for (int k = 0; k < 4; ++k) s += lsum[wg * 4 + k][tid];
        KvRowOut o = {0.f, 0.f, nullptr, nullptr, nullptr};
        if (q < n_q && q - r * p.gw < gw) o = out(q, r, s == 0.f ? kNegInf : sm.ref[q] * c, s, true);
        outs[q] = o;
      }
      named_bar_sync(bar, 128);
      const int d = wq * 32 + lane;
      const bool final_row = whole && p.put_o == nullptr;
      float odd = 0.f;                       // NaN after a value that is not finite
      // Sums and prefixes leave as they lie, 128 bytes a warp's store; final rows go through shared memory (this
      // group's share of the weights' place, kW queries at a time), into packs of 16 bytes.
      E* stage = reinterpret_cast<E*>(ps + kEndBytes + wg * kStageBytes);
#pragma unroll 1
      for (int k0 = 0; k0 < kOwn && q0 + k0 < n_q; k0 += kW) {
        uint32_t s[16];
        tmem_ld16(lanes + 2 * kNQ + q0 + k0, s);
        tmem_ld_wait();
        reg_fence(s);
#pragma unroll
        for (int k = 0; k < kW; ++k) odd = fmaf(0.f, d < dim && q0 + k0 + k < n_q ? __uint_as_float(s[k]) : 0.f, odd);
        if (!final_row) {
#pragma unroll
          for (int k = 0; k < kW; ++k) {
            float* to = outs[q0 + k0 + k].dst_f;
            if (q0 + k0 + k < n_q && to != nullptr && d < dim) to[d] = __uint_as_float(s[k]);
          }
          continue;
        }
        if (p.pre_o != nullptr) {
#pragma unroll
          for (int k = 0; k < kW; ++k) {
            const KvRowOut& o = outs[q0 + k0 + k];
            const float pre = q0 + k0 + k < n_q && o.dst != nullptr && d < dim ? o.pre[d] * o.f_pre : 0.f;
            s[k] = __float_as_uint(fmaf(__uint_as_float(s[k]), o.f, pre));
          }
        } else {
#pragma unroll
          for (int k = 0; k < kW; ++k) s[k] = __float_as_uint(__uint_as_float(s[k]) * outs[q0 + k0 + k].f);
        }
#pragma unroll
        for (int k = 0; k < kW; ++k)
          if (d < C::kChunks * 64) stage[k * (C::kChunks * 64) + d] = E(__uint_as_float(s[k]));
        named_bar_sync(bar, 128);
        const int packs = dim / 8;
        for (int i = tid; i < kW * packs; i += 128) {
          const int k = i / packs, c = i - k * packs;
          E* to = q0 + k0 + k < n_q ? static_cast<E*>(outs[q0 + k0 + k].dst) : nullptr;
          if (to != nullptr)
            reinterpret_cast<uint4*>(to)[c] = reinterpret_cast<const uint4*>(stage + k * (C::kChunks * 64))[c];
        }
        named_bar_sync(bar, 128);
      }
      if (!(odd == 0.f)) mi.odd = 1;
      tc_fence_before();
      named_bar_sync(kAllBar, kAll);
      if (opens && threadIdx.x == 0) {
        cut = make_int4(tile_id, unit, mi.line.last_before(mi.line.start(id + 1) + (tile.nb - b1)) - id + 1, 0);
      }
    }
    if (threadIdx.x == 0 && count > 0) p.cuts[id] = cut;
    // Results that are not finite are taken again here, when no role waits for this one any more: the time
    // that it takes is bounded by nothing but the tokens, and a wait gives up after a limit.
    if (count > 0 && mi.odd != 0 && !*ab.smem) take_odd_again<E, C::kChunks * 64>(p, mi.start[0], count, id, warp, kSoftWarps);
  }
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc(tmem, C::kCols);
  pdl_release();
}

template <class C>
cudaError_t run_tc(KvPass& p, const KvMaps& maps, int sms, int* status, cudaStream_t s) {
  static_assert(smem_bytes<C>() <= 227 * 1024, "fits an SM");
  static_assert(end_bytes<C>() + C::kGroups * stage_bytes<C>() <= C::kPBytes * C::kPBufs,
                "an item's end reuses the weights' place");
  shape_pass(p, C::kNQ, 32, kBlk);
  p.block_workers = 1;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_smem(kv_tc_kernel<C>, int(smem_bytes<C>()), done);
  if (e != cudaSuccess) return e;
  return launch_pdl(kv_tc_kernel<C>, dim3(std::min(sms, kKvMostSms)), dim3(C::kThreads), smem_bytes<C>(), s,
                    maps, p, status);
}

}  // namespace

cudaError_t launch_kv_tc(KvPass& p, const KvMaps& maps, int sms, int* status, cudaStream_t s) {
  const int group = p.a.H / p.a.c.heads;
  const long long queries = std::min<long long>(std::min<long long>(p.part.per, p.a.N), 32) * group;
  if (p.a.c.dim <= 64)
    return queries <= 64 ? run_tc<Cfg<64, 1>>(p, maps, sms, status, s) : run_tc<Cfg<128, 1>>(p, maps, sms, status, s);
  return queries <= 64 ? run_tc<Cfg<64, 2>>(p, maps, sms, status, s) : run_tc<Cfg<128, 2>>(p, maps, sms, status, s);
}

}  // namespace alr
