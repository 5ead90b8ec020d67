// The paged key-value cache: the step's block tables and slot map, and new rows into their slots.
#include <algorithm>

#include "kernels.h"
#include "launch.h"
#include "row_reduce.cuh"

namespace alr {
namespace {

// ------------------------------------------------------------------------ plan ---
// Everything follows from sums over the sequences before one: of the tokens asked for (its first row of
// the batch), of the new pages (its place in the list of free pages) and of the returned ones (theirs).
// Each block takes those sums over all sequences for itself (S is at most 8192, 8 KB a thousand).  A
// token's page is found from its sequence's sums, be it an old one, one out of the pool or one that
// another sequence returns in this step, so blocks share rows and pages and none reads what another
// writes.  Lengths and the pool's count may be updated in place: one block does everything where rows are
// few, else a second launch writes them.
//   Bound by latency: two loads, two scans, two dependent loads a token (768 rows of 768 sequences: 12 us a call
// in a loop of calls, of which the host takes 11; 393 thousand rows of 96 prompts: 15, by one cluster of 8
// blocks that shared all the writing 47).
constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;

// Sums of the threads before this one (v becomes that), and of all.  buf: kPlanWarps entries, free
// again on return.
ALR_DEV long long scan_before(long long& v, long long* buf) {
  const long long own = v, up = warp_scan(v);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 31) buf[warp] = up;
  __syncthreads();
  const long long w = warp_scan(lane < kPlanWarps ? buf[lane] : 0ll);
  const long long before = warp == 0 ? 0ll : __shfl_sync(0xffffffffu, w, warp - 1);
  const long long all = __shfl_sync(0xffffffffu, w, kPlanWarps - 1);
  __syncthreads();
  v = before + up - own;
  return all;
}

// Largest i in [0, n) with a[i] <= k: the entry that element k of the running sums a[0] = 0 <= a[1] <= ...
// belongs to (the last of those with the same sum, which is the one that is not empty).
ALR_DEV int owner_of(const int* a, int n, int k) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= k) lo = mid;
    else hi = mid;
  }
  return lo;
}

struct PlanSums {
  int* start;   // [S + 1] first row of the batch (at most T)
  int* len;     // [S] tokens held; ~tokens where the rows get no slot (refused or ended)
  int* fresh;   // [S] new pages before
  int* back;    // [S] returned pages before
};

ALR_DEV int pages_of(long long tokens, int page) { return int((tokens + page - 1) / page); }

// rows: write rows, tables and the pool (blocks share them); sums: lengths, starts and counts (one block).
__global__ void __launch_bounds__(kPlanThreads) kv_plan_kernel(const KvPlan p, bool rows, bool sums) {
  extern __shared__ int plan_smem[];
  __shared__ long long buf[kPlanWarps];
  const int S = p.S, tid = threadIdx.x, rank = blockIdx.x, n_cta = gridDim.x;
  const PlanSums t = {plan_smem, plan_smem + S + 1, plan_smem + 2 * S + 1, plan_smem + 3 * S + 1};
  pdl_wait_and_release();
  const int used = min(max(*p.pool_used, 0), p.n_pool);
  const long long most = (long long)p.cols * p.page;
  const int per = (S + kPlanThreads - 1) / kPlanThreads;
  const int s0 = min(tid * per, S), s1 = min(s0 + per, S);

  long long tokens = 0, back = 0;
  for (int s = s0; s < s1; ++s) {
    const int n = int(min((long long)max(p.len[s], 0), most)), a = p.add[s];
    t.len[s] = n;
    t.back[s] = int(min(back, (long long)INT32_MAX));
    t.start[s] = a;                          // for now
    tokens += max(a, 0);
    if (a < 0) back += pages_of(n, p.page);
  }
  long long before = tokens, back_before = back;
  const long long all = scan_before(before, buf);
  const long long n_back = scan_before(back_before, buf);
  const long long n_free = p.n_pool - used + n_back;
  long long need = 0, row = before;
  for (int s = s0; s < s1; ++s) {
    const int a = t.start[s], n = t.len[s];
    if (a >= 0 && n + (long long)a <= most && row + a <= p.T)
      need += pages_of(n + (long long)a, p.page) - pages_of(n, p.page);
    row += max(a, 0);
  }
  long long need_before = need;
  scan_before(need_before, buf);
  // the sequences' answers; n_new: the pages that are taken, up to the last sequence that gets any
  int refused = 0;
  long long k = need_before, n_new = 0;
  row = before;
  __syncthreads();                           // len and pool_used have been read: they may be written
  for (int s = s0; s < s1; ++s) {
    const int a = t.start[s], n = t.len[s];
    const bool asks = a >= 0 && n + (long long)a <= most && row + a <= p.T;
    const int w = asks ? pages_of(n + (long long)a, p.page) - pages_of(n, p.page) : 0;
    const bool ok = asks && (w == 0 || k + w <= n_free);
    t.back[s] = int(min(back_before + t.back[s], (long long)INT32_MAX));
    t.fresh[s] = int(min(k, (long long)INT32_MAX));
    t.start[s] = int(min(row, (long long)p.T));
    if (!ok) t.len[s] = ~n;
    if (a >= 0 && !ok) ++refused;
    if (ok && w > 0) n_new = k + w;
    if (sums) {
      p.out_len[s] = a < 0 ? 0 : ok ? n + a : n;
      if (p.start != nullptr) p.start[s] = int(min(row, (long long)INT32_MAX));
    }
    k += w;
    row += max(a, 0);
  }
  const int n_rows = int(min(all, (long long)p.T));
  if (tid == 0) {
    t.start[S] = n_rows;
    if (sums && p.start != nullptr) p.start[S] = int(min(all, (long long)INT32_MAX));
  }
  n_new = block_reduce(n_new, MaxOp(), buf);
  if (sums) {
    const long long r = block_reduce((long long)refused, AddOp(), buf);
    if (tid == 0) {
      *p.out_used = int(max(used - n_back + n_new, 0ll));
      if (p.n_refused != nullptr) *p.n_refused = int(r);
    }
  }
  if (!rows) return;
  __syncthreads();

  // page number i of the list of free pages: the returned ones, then the pool's
  const auto returned = [&](int i) {
    const int s = owner_of(t.back, S, i);
    return p.table[(long long)s * p.cols + (i - t.back[s])];
  };
  const auto page_at = [&](int i) {
    return i < n_back ? returned(i) : p.pool[used + (i - int(n_back))];
  };
  const int first = rank * kPlanThreads + tid, step = n_cta * kPlanThreads;
  for (long long i = first; i < n_back; i += step) {
    const long long at = used - n_back + i;
    if (at >= 0) p.pool[at] = returned(int(i));
  }
  for (long long i = first; i < n_new; i += step) {
    const int s = owner_of(t.fresh, S, int(i));
    const int n = t.len[s] < 0 ? ~t.len[s] : t.len[s];
    p.table[(long long)s * p.cols + pages_of(n, p.page) + (int(i) - t.fresh[s])] = page_at(int(i));
  }
  // rows: one each where there are threads for all (a step of single tokens), else each warp has a stretch of
  // its own, whose sequences follow one another, a lane four rows at a time, which mostly lie in one page
  const int n_warps = n_cta * kPlanWarps, stretch = ((p.T - 1) / n_warps + 128) / 128 * 128;   // T up to 2^31 - 1
  const long long r0 = (long long)(rank * kPlanWarps + (tid >> 5)) * stretch;
  int s = -1;
  const auto owner = [&](int r) {            // sequence of row r < n_rows, searched from the last one on
    if (s >= 0 && r >= t.start[s] && r < t.start[s + 1]) return s;
    int i = s < 0 || r < t.start[s] ? S : s + 1;
    for (int c = 0; c < 4 && i < S && r >= t.start[i + 1]; ++c) ++i;
    return i < S && r < t.start[i + 1] ? i : owner_of(t.start, S, r);
  };
  const auto slot_at = [&](int pg, int off) {
    const long long at = (long long)pg * p.page + off;
    return pg < 0 || at > INT32_MAX ? -1 : int(at);
  };
  const auto page_of = [&](int q, int j) {   // the j-th page of sequence q
    const int old = pages_of(t.len[q], p.page);
    return j < old ? p.table[(long long)q * p.cols + j] : page_at(t.fresh[q] + (j - old));
  };
  if (p.T <= n_cta * kPlanThreads) {
    const int r = rank * kPlanThreads + tid;
    if (r >= p.T) return;
    int slot = -1, seq = -1, n = 0;
    if (r < n_rows) {
      s = owner_of(t.start, S, r);
      if (t.len[s] >= 0) {
        const int at = t.len[s] + r - t.start[s], k = at / p.page;
        seq = s;
        n = at + 1;
        slot = slot_at(page_of(s, k), at - k * p.page);
      }
    }
    p.slot[r] = slot;
    if (p.tok_seq != nullptr) p.tok_seq[r] = seq;
    if (p.tok_len != nullptr) p.tok_len[r] = n;
    return;
  }
  for (long long r = r0 + 4 * (tid & 31); r < min(r0 + stretch, (long long)p.T); r += 128) {
    int slot[4] = {-1, -1, -1, -1}, seq[4] = {-1, -1, -1, -1}, n[4] = {};
    if (r < n_rows) {
      s = owner(int(r));
      const int held = t.len[s], pos = held + int(r) - t.start[s], j = pos / p.page, off = pos - j * p.page;
      if (r + 3 < t.start[s + 1] && off + 3 < p.page) {
        if (held >= 0) {
          const int first = slot_at(page_of(s, j), off);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            seq[e] = s;
            n[e] = pos + e + 1;
            slot[e] = first < 0 ? -1 : first + e;
          }
        }
      } else {
#pragma unroll 1
        for (int e = 0; e < 4 && r + e < n_rows; ++e) {
          s = owner(int(r) + e);
          if (t.len[s] < 0) continue;
          const int at = t.len[s] + int(r) + e - t.start[s], k = at / p.page;
          seq[e] = s;
          n[e] = at + 1;
          slot[e] = slot_at(page_of(s, k), at - k * p.page);
        }
      }
    }
    const auto put = [&](int32_t* to, const int (&v)[4]) {
      if (to == nullptr) return;
      if (p.packs && r + 3 < p.T) {
        *reinterpret_cast<int4*>(to + r) = make_int4(v[0], v[1], v[2], v[3]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (r + e < p.T) to[r + e] = v[e];
      }
    };
    put(p.slot, slot);
    put(p.tok_seq, seq);
    put(p.tok_len, n);
  }
}

// ---------------------------------------------------------------------- append ---
// Memory-bound: a warp moves 32 kAppendBatch packs of 16 bytes (of the cache) of one token, its keys' and
// values' rows one after the other, all loads issued before the stores (32768 tokens of 4 x 128 bf16: 19.7 us,
// 6.2 TB/s; with a warp for the keys and one for the values, half their loads beyond the row, 24.4).
constexpr int kAppendThreads = 256;
constexpr int kAppendBatch = 4;

// magic: q / packs is the high word of q * magic (exact for q * packs < 2^32).
template <typename E, typename F>
__global__ void __launch_bounds__(kAppendThreads)
    kv_append_kernel(const KvCache c, const F* k_new, const F* v_new, long long T, long long ld,
                     const int32_t* slot, int pieces, uint32_t magic) {
  constexpr int kPack = 16 / sizeof(E);
  // A pack of the new rows is as aligned as it is long, up to 16 bytes: of bf16 for an fp32 cache 8, of fp32 for a
  // bf16 cache 32 at 16.
  constexpr int kSrcBytes = kPack * int(sizeof(F));
  struct alignas(16) Dst { E e[kPack]; };
  struct alignas(kSrcBytes < 16 ? kSrcBytes : 16) Src { F e[kPack]; };
  static_assert(sizeof(Dst) == 16 && sizeof(Src) == kSrcBytes, "a pack's elements and nothing behind them");
  pdl_wait_and_release();
  const long long w = (long long)blockIdx.x * (kAppendThreads / 32) + threadIdx.x / 32;
  const long long i = pieces == 1 ? w : w / pieces;
  if (i >= T) return;
  const int at = slot[i];
  if (at < 0 || at >= (long long)c.n_pages * c.page) return;
  const int packs = c.dim / kPack, row = c.heads * packs;
  const int first = int(w - i * pieces) * 32 * kAppendBatch + (threadIdx.x & 31);
  const int pg = at / c.page;
  const long long to = pg * c.sp + (at - pg * c.page) * c.st;
  Src x[kAppendBatch];
#pragma unroll
  for (int j = 0; j < kAppendBatch; ++j) {
    const int q = first + 32 * j;
    const F* src = (q < row ? k_new : v_new) + i * ld + (q < row ? q : q - row) * kPack;
    if (q < 2 * row) x[j] = *reinterpret_cast<const Src*>(src);
  }
#pragma unroll
  for (int j = 0; j < kAppendBatch; ++j) {
    const int q = first + 32 * j, r = q < row ? q : q - row;
    if (q >= 2 * row) break;
    const int head = packs == 1 ? r : int(__umulhi(uint32_t(r), magic));
    Dst y;
#pragma unroll
    for (int e = 0; e < kPack; ++e) y.e[e] = E(to_float(x[j].e[e]));
    E* dst = static_cast<E*>(q < row ? c.K : c.V) + to + head * c.sh + (r - head * packs) * kPack;
    *reinterpret_cast<Dst*>(dst) = y;
  }
}

template <typename E, typename F>
cudaError_t run_append(const KvCache& c, const void* K_new, const void* V_new, long long T,
                       long long ld, const int32_t* slot, cudaStream_t s) {
  const int packs = c.dim / int(16 / sizeof(E)), row = c.heads * packs;
  const int pieces = (2 * row + 32 * kAppendBatch - 1) / (32 * kAppendBatch);
  const long long warps = T * pieces, per = kAppendThreads / 32;
  if ((warps + per - 1) / per > INT32_MAX) return cudaErrorInvalidConfiguration;
  const uint32_t magic = packs == 1 ? 0 : uint32_t(((uint64_t(1) << 32) + packs - 1) / packs);
  return launch_pdl(kv_append_kernel<E, F>, dim3(unsigned((warps + per - 1) / per)),
                    dim3(kAppendThreads), 0, s, c, static_cast<const F*>(K_new),
                    static_cast<const F*>(V_new), T, ld, slot, pieces, magic);
}

}  // namespace

cudaError_t launch_kv_plan(KvPlan p, cudaStream_t s) {
  const auto packs = [](const void* x) { return (reinterpret_cast<uintptr_t>(x) & 15) == 0; };
  p.packs = packs(p.slot) && packs(p.tok_seq) && packs(p.tok_len);
  const size_t smem = size_t(4 * p.S + 1) * sizeof(int);
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_smem(kv_plan_kernel, int((4 * kKvMaxSeqs + 1) * sizeof(int)), done);
  if (e != cudaSuccess) return e;
  const int n_cta = int(std::min((p.T + 4095ll) / 4096, 128ll));
  if (n_cta <= 1) return launch_pdl(kv_plan_kernel, dim3(1), dim3(kPlanThreads), smem, s, p, true, true);
  const cudaError_t f = launch_pdl(kv_plan_kernel, dim3(n_cta), dim3(kPlanThreads), smem, s, p, true, false);
  return f != cudaSuccess ? f
                          : launch_pdl(kv_plan_kernel, dim3(1), dim3(kPlanThreads), smem, s, p, false, true);
}

cudaError_t launch_kv_append(const KvCache& c, const void* K_new, const void* V_new, int src_dtype,
                             long long T, long long ld, const int32_t* slot, cudaStream_t s) {
  using B = __nv_bfloat16;
  if (c.dtype == 0)
    return src_dtype == 0 ? run_append<B, B>(c, K_new, V_new, T, ld, slot, s)
                          : run_append<B, float>(c, K_new, V_new, T, ld, slot, s);
  return src_dtype == 0 ? run_append<float, B>(c, K_new, V_new, T, ld, slot, s)
                        : run_append<float, float>(c, K_new, V_new, T, ld, slot, s);
}

}  // namespace alr
