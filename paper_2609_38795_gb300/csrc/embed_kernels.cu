// Embedding of tokens, scaled, and the gradient of the table by sorted tokens.
#include <algorithm>

#include "kernels.h"
#include "launch.h"
#include "row_reduce.cuh"

namespace alr {
namespace {

// kCols consecutive elements of a row as one load or store (16 bytes at most).
template <typename E, int kCols>
struct alignas(sizeof(E) * kCols) Pack {
  E e[kCols];
};

// ---------------------------------------------------------------------- lookup ---
// out[i] = scale * E[token_i] (fp32 product, rounded once); a token outside [0, V) gives zeros.
// Memory-bound: a warp moves 32 kEmbedBatch packs of one row, all loads issued before the stores
// (32768 x 4096 bf16 rows, 15 of 16 the same token: 43.5 us, 6.55 TB/s).
constexpr int kEmbedThreads = 256;
constexpr int kEmbedBatch = 8;

template <typename E, int kCols>
__global__ void __launch_bounds__(kEmbedThreads)
    embed_kernel(const E* table, int V, int packs, int pieces, const int32_t* tokens, long long N,
                 float scale, E* out) {
  using P = Pack<E, kCols>;
  pdl_wait_and_release();
  const long long w = (long long)blockIdx.x * (kEmbedThreads / 32) + threadIdx.x / 32;
  const long long i = w / pieces;
  if (i >= N) return;
  const int first = int(w - i * pieces) * 32 * kEmbedBatch + (threadIdx.x & 31);
  const int v = tokens[i];
  const bool ok = v >= 0 && v < V;
  const P* src = reinterpret_cast<const P*>(table) + (ok ? (long long)v * packs : 0);
  P* dst = reinterpret_cast<P*>(out) + i * packs;
  P x[kEmbedBatch];
#pragma unroll
  for (int j = 0; j < kEmbedBatch; ++j)
    if (ok && first + 32 * j < packs) x[j] = src[first + 32 * j];
#pragma unroll
  for (int j = 0; j < kEmbedBatch; ++j) {
    if (first + 32 * j >= packs) break;
#pragma unroll
    for (int c = 0; c < kCols; ++c) x[j].e[c] = ok ? E(to_float(x[j].e[c]) * scale) : E(0.f);
    dst[first + 32 * j] = x[j];
  }
}

// -------------------------------------------------------------------- gradient ---
// dE[v] = scale * sum of dY's rows of token v.  The rows are ordered by token (a stable radix sort),
// cut into chunks of P rows whatever their tokens are, and a block adds up its chunk's runs of equal
// tokens: the work is the same for one token in every row as for as many tokens as rows, and no
// atomic decides an order.
//   A run of at most P rows belongs to the chunk that it starts in, which follows it into the
// next one and writes the table's row.  A longer run leaves one partial sum in each chunk that it
// touches, and a last kernel adds those in order.
//   32768 x 2048 bf16 rows into a 32000-token fp32 table, 15 of 16 rows one token: 101 us; sort 21 (latency of
// its two passes on 8 SMs), chunks and the zeros of absent tokens 66 (396 MB, 6 TB/s), join 12.  The zeros
// written beside the sort instead, by blocks that look up their rows themselves: 149 us.
// Few rows take one kernel instead, in which the block of each row looks for its token's others (192 rows
// with their lookup: 12 us, two launches, most of it the host's two calls).

template <typename E, int kCols>
ALR_DEV void add_pack(float (&acc)[kCols], const Pack<E, kCols>& x) {
#pragma unroll
  for (int c = 0; c < kCols; ++c) acc[c] += to_float(x.e[c]);
}

// A finished sum into the table's row (or a partial sum's): written by packs of 16 bytes at most.
template <int kCols>
ALR_DEV void put_sum(float* dst, const float (&acc)[kCols], float scale, bool accumulate) {
  constexpr int kW = kCols < 4 ? kCols : 4;
  using P = Pack<float, kW>;
#pragma unroll
  for (int c = 0; c < kCols; c += kW) {
    P* p = reinterpret_cast<P*>(dst + c);
    P v = {};
    if (accumulate) v = *p;
#pragma unroll
    for (int k = 0; k < kW; ++k) v.e[k] = fmaf(scale, acc[c + k], v.e[k]);
    *p = v;
  }
}

// Zeros in the table rows [v0, v0 + n) whose bit in `present` is clear (whole block).
ALR_DEV void zero_rows(float* dE, int d, int v0, int n, const uint32_t* present) {
  for (int k = 0; k < n; ++k) {
    if (present[k >> 5] >> (k & 31) & 1) continue;
    float* row = dE + (long long)(v0 + k) * d;
    if (d % 4 == 0)
      for (int c = threadIdx.x; c < d / 4; c += blockDim.x)
        reinterpret_cast<float4*>(row)[c] = make_float4(0.f, 0.f, 0.f, 0.f);
    else
      for (int c = threadIdx.x; c < d; c += blockDim.x) row[c] = 0.f;
  }
}

// --- few rows: one kernel.  Blocks [0, N * slices) take a row and a slice of `lanes` packs of its
// columns: the first row of each token gathers all rows of it, each group of `lanes` threads taking
// every (kFewThreads / lanes)-th one.  The other blocks zero the table rows of absent tokens.
constexpr int kFewRows = 512;
constexpr int kFewThreads = 256;

template <typename E, int kCols>
__global__ void __launch_bounds__(kFewThreads)
    embed_grad_few_kernel(const E* dY, int V, int d, const int32_t* tokens, int N, int slices,
                          int lanes, float scale, int accumulate, float* dE) {
  __shared__ int tok[kFewRows];
  __shared__ int rows[kFewRows];
  __shared__ float sums[kFewThreads * kCols];
  __shared__ int n_rows, earlier;
  __shared__ uint32_t present;
  pdl_wait_and_release();
  if (threadIdx.x == 0) {
    present = 0;
    earlier = 0;
  }
  for (int j = threadIdx.x; j < N; j += kFewThreads) tok[j] = tokens[j];
  __syncthreads();
  if (int(blockIdx.x) >= N * slices) {
    const int v0 = (int(blockIdx.x) - N * slices) * 32;
    for (int j = threadIdx.x; j < N; j += kFewThreads)
      if (tok[j] >= v0 && tok[j] - v0 < 32) atomicOr(&present, 1u << (tok[j] - v0));
    __syncthreads();
    zero_rows(dE, d, v0, min(32, V - v0), &present);
    return;
  }
  const int i = blockIdx.x / slices, slice = blockIdx.x - i * slices, v = tok[i];
  if (v < 0 || v >= V) return;
  for (int j = threadIdx.x; j < i; j += kFewThreads)
    if (tok[j] == v) earlier = 1;
  __syncthreads();
  if (earlier) return;
  if (threadIdx.x < 32) {   // the token's rows, in order
    int n = 0;
    for (int j0 = i; j0 < N; j0 += 32) {
      const int j = j0 + threadIdx.x;
      const bool is = j < N && tok[j] == v;
      const unsigned ball = __ballot_sync(0xffffffffu, is);
      if (is) rows[n + __popc(ball & ((1u << threadIdx.x) - 1u))] = j;
      n += __popc(ball);
    }
    if (threadIdx.x == 0) n_rows = n;
  }
  __syncthreads();
  const int group = threadIdx.x / lanes, lane = threadIdx.x % lanes, groups = kFewThreads / lanes;
  const int pack = slice * lanes + lane, packs = d / kCols, n = n_rows;
  float acc[kCols] = {};
  if (pack < packs) {
#pragma unroll 8
    for (int k = group; k < n; k += groups)
      add_pack(acc, reinterpret_cast<const Pack<E, kCols>*>(dY)[(long long)rows[k] * packs + pack]);
  }
  if (n > 1) {
#pragma unroll
    for (int c = 0; c < kCols; ++c) sums[c * kFewThreads + threadIdx.x] = acc[c];
    __syncthreads();
    if (group == 0)
      for (int g = 1; g < min(groups, n); ++g)
#pragma unroll
        for (int c = 0; c < kCols; ++c) acc[c] += sums[c * kFewThreads + g * lanes + lane];
  }
  if (group == 0 && pack < packs)
    put_sum(dE + (long long)v * d + pack * kCols, acc, scale, accumulate != 0);
}

// --- stable radix sort of (token, row) by one cluster: each warp ranks the keys of its own
// stretch of rows, so equal tokens stay in row order.  Tokens outside [0, V) get the key V.
constexpr int kSortThreads = 512;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortCtas = 8;
constexpr int kSortBits = 9;            // of the key at most in a pass
constexpr int kSortBins = 1 << kSortBits;
constexpr int kSortBatch = 8;           // steps of 32 keys that a warp has in flight

// Lanes that hold the same digit (the keys past the end, all ones, differ from any digit in the bit
// above).  A ballot for each bit: a match instruction takes a turn for each distinct value (the first
// sweep over 32768 tokens of a 32000-token table 11.5 K cycles with it, 6.6 K with ballots).
ALR_DEV unsigned digit_peers(uint32_t digit, int bits) {
  unsigned peers = 0xffffffffu;
#pragma unroll
  for (int b = 0; b <= kSortBits; ++b) {
    if (b > bits) break;
    const unsigned set = __ballot_sync(0xffffffffu, digit >> b & 1);
    peers &= digit >> b & 1 ? set : ~set;
  }
  return peers;
}

struct GradPlan {
  int chunk, n_chunks, passes, bits;
  size_t tok_off[2], row_off[2], list_off, count_off, present_off, part_off, total;
};

// Rows of a chunk: enough chunks to fill the device, few partial sums for a token in every row (4000 rows:
// 61.6 us at 16, 61.1 at 32; 12000: 74 at 32, 79 at 16; 32768: 102 at 64, 110 at 32; 100000: 202 at 128, 207 at 64).
GradPlan grad_plan(int V, int d, int N) {
  GradPlan g{};
  g.chunk = N <= 8192 ? 16 : N <= 16384 ? 32 : N <= 65536 ? 64 : 128;
  g.n_chunks = (N + g.chunk - 1) / g.chunk;
  int bits = 1;
  while ((long long)V >> bits != 0) ++bits;    // keys 0 .. V
  g.passes = (bits + kSortBits - 1) / kSortBits;
  g.bits = (bits + g.passes - 1) / g.passes;
  size_t at = 0;
  auto take = [&at](size_t bytes) {
    const size_t off = at;
    at += (bytes + 255) / 256 * 256;
    return off;
  };
  for (int k = 0; k < 2; ++k) {
    g.tok_off[k] = take(size_t(N) * 4);
    g.row_off[k] = take(size_t(N) * 4);
  }
  g.list_off = take(size_t(g.n_chunks) * 8);
  g.count_off = take(4);
  g.present_off = take((size_t(V) + 31) / 32 * 4);
  g.part_off = take(size_t(g.n_chunks) * 2 * d * sizeof(float));
  g.total = at;
  return g;
}

// Also: `present`, a bit for each token that occurs (nullptr: not wanted), and the runs of more than
// `chunk` rows in `list` (first place in the order and token, in any order), their number in *count.
__global__ void __launch_bounds__(kSortThreads)
    embed_sort_kernel(const int32_t* tokens, int N, int V, int passes, int bits, int chunk,
                      uint32_t* tok0, uint32_t* row0, uint32_t* tok1, uint32_t* row1,
                      uint32_t* present, int2* list, int32_t* count) {
  __shared__ uint32_t hist[kSortWarps][kSortBins];
  __shared__ uint32_t cta_total[kSortBins];
  __shared__ uint32_t scan[kSortWarps];
  pdl_wait_and_release();
  const int rank = int(cluster_ctarank()), warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const int all = kSortCtas * kSortThreads, me = rank * kSortThreads + int(threadIdx.x);
  if (present != nullptr)
    for (int i = me; i < (V + 31) / 32; i += all) present[i] = 0;
  if (me == 0) *count = 0;
  // this warp's stretch, in steps of 32
  const int steps = (N + 32 * kSortCtas * kSortWarps - 1) / (32 * kSortCtas * kSortWarps);
  const int begin = (rank * kSortWarps + warp) * steps * 32;
  const int bins = 1 << bits;
  uint32_t *src_t = nullptr, *src_r = nullptr, *dst_t = tok0, *dst_r = row0;
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * bits;
    const uint32_t* keys = pass > 0 ? src_t : reinterpret_cast<const uint32_t*>(tokens);
    // keys (and rows) of kSortBatch steps, all loads in flight; ~0 past the end
    auto load = [&](int s0, uint32_t (&key)[kSortBatch], uint32_t (&row)[kSortBatch], bool rows) {
#pragma unroll
      for (int j = 0; j < kSortBatch; ++j) {
        const int p = min(begin + (s0 + j) * 32 + lane, N - 1);
        key[j] = __ldcg(keys + p);
        row[j] = uint32_t(p);
      }
      if (rows && pass > 0)
#pragma unroll
        for (int j = 0; j < kSortBatch; ++j) row[j] = __ldcg(src_r + row[j]);
#pragma unroll
      for (int j = 0; j < kSortBatch; ++j) {
        if (key[j] >= uint32_t(V)) key[j] = uint32_t(V);   // first pass: outside [0, V)
        if (s0 + j >= steps || begin + (s0 + j) * 32 + lane >= N) key[j] = 0xffffffffu;
      }
    };
    for (int b = lane; b < bins; b += 32) hist[warp][b] = 0;
    __syncwarp();
    uint32_t key[kSortBatch], row[kSortBatch];
    for (int s0 = 0; s0 < steps; s0 += kSortBatch) {
      load(s0, key, row, false);
#pragma unroll
      for (int j = 0; j < kSortBatch; ++j) {
        if (s0 + j >= steps) break;
        const uint32_t digit =
            key[j] != 0xffffffffu ? (key[j] >> shift) & (bins - 1) : 0xffffffffu;
        const unsigned peers = digit_peers(digit, bits);
        if (digit != 0xffffffffu && (peers >> lane) == 1u) hist[warp][digit] += __popc(peers);
        __syncwarp();
      }
    }
    __syncthreads();
    // offsets: of the digit, of this block within it, of each warp within the block
    uint32_t mine = 0;
    const int b = threadIdx.x;
    if (b < bins) {
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t n = hist[w][b];
        hist[w][b] = mine;
        mine += n;
      }
      cta_total[b] = mine;
    }
    cluster_sync();
    uint32_t before = 0, total = 0;
    if (b < bins) {
#pragma unroll
      for (int c = 0; c < kSortCtas; ++c) {
        const uint32_t n = uint32_t(ld_cluster_s32(cluster_smem_addr(&cta_total[b], uint32_t(c))));
        if (c < rank) before += n;
        total += n;
      }
    }
    uint32_t incl = warp_scan(total);
    if (lane == 31) scan[warp] = incl;
    __syncthreads();
    for (int w = 0; w < warp; ++w) incl += scan[w];
    const uint32_t base = incl - total + before;
    if (b < bins)
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) hist[w][b] += base;
    __syncthreads();
    for (int s0 = 0; s0 < steps; s0 += kSortBatch) {
      load(s0, key, row, true);
#pragma unroll
      for (int j = 0; j < kSortBatch; ++j) {
        if (s0 + j >= steps) break;
        const bool in = key[j] != 0xffffffffu;
        const uint32_t digit = in ? (key[j] >> shift) & (bins - 1) : 0xffffffffu;
        const unsigned peers = digit_peers(digit, bits);
        const bool last = in && (peers >> lane) == 1u;
        uint32_t at = 0;
        if (in) {
          at = hist[warp][digit] + __popc(peers & ((1u << lane) - 1u));
          dst_t[at] = key[j];
          dst_r[at] = row[j];
        }
        __syncwarp();
        if (last) hist[warp][digit] = at + 1;
        __syncwarp();
      }
    }
    cluster_sync();   // the sorted pairs are written; cta_total may be overwritten
    src_t = dst_t;
    src_r = dst_r;
    dst_t = src_t == tok0 ? tok1 : tok0;
    dst_r = src_r == row0 ? row1 : row0;
  }
#pragma unroll 4
  for (int p = me; p < N; p += all) {
    const uint32_t t = __ldcg(src_t + p), before = p > 0 ? __ldcg(src_t + p - 1) : 0xffffffffu;
    const uint32_t far = p + chunk < N ? __ldcg(src_t + p + chunk) : 0xffffffffu;
    if (t >= uint32_t(V) || t == before) continue;   // no token's first row
    if (present != nullptr) atomicOr(present + (t >> 5), 1u << (t & 31));
    if (far == t) list[atomicAdd(count, 1)] = make_int2(p, int(t));
  }
}

// --- sums of a chunk's runs (blocks [0, n_chunks * slices): a chunk and a slice of the columns),
// zeros for absent tokens (the others).
constexpr int kChunkThreads = 256;
constexpr int kChunkMost = 128;
constexpr int kChunkBatch = 8;

template <typename E, int kCols>
__global__ void __launch_bounds__(kChunkThreads)
    embed_chunk_kernel(const E* dY, int V, int d, const uint32_t* tok_s, const uint32_t* row_s, int N,
                       int chunk, int n_chunks, int slices, float scale, int accumulate, float* dE,
                       float* part, const uint32_t* present) {
  // tokens of the chunk, of as many rows before and after it; ~0 outside
  __shared__ uint32_t tok[3 * kChunkMost];
  __shared__ uint32_t row[2 * kChunkMost];
  __shared__ int back, lead_end, trail, trail_end, valid_end;
  pdl_wait_and_release();
  if (int(blockIdx.x) >= n_chunks * slices) {
    const int g = int(blockIdx.x) - n_chunks * slices;
    zero_rows(dE, d, g * 32, min(32, V - g * 32), present + g);
    return;
  }
  const int c = blockIdx.x / slices, slice = blockIdx.x - c * slices;
  const int p0 = c * chunk, n = min(chunk, N - p0), tid = threadIdx.x;
  if (tid == 0) {
    back = chunk;
    lead_end = trail_end = valid_end = 2 * chunk;
    trail = 0;
  }
  for (int k = tid; k < 3 * chunk; k += kChunkThreads) {
    const int p = p0 - chunk + k;
    tok[k] = p >= 0 && p < N ? tok_s[p] : 0xffffffffu;
  }
  for (int k = tid; k < 2 * chunk; k += kChunkThreads) row[k] = p0 + k < N ? row_s[p0 + k] : 0u;
  __syncthreads();
  const uint32_t* t = tok + chunk;   // t[k]: token of row p0 + k in the order
  const uint32_t first = t[0], last = t[n - 1];
  for (int k = tid; k < 2 * chunk; k += kChunkThreads) {
    if (k < chunk && t[-1 - k] != first) atomicMin(&back, k);
    if (t[k] != first) atomicMin(&lead_end, k);
    if (k >= n && t[k] != last) atomicMin(&trail_end, k);
    if (k > 0 && k < n && t[k] != t[k - 1]) atomicMax(&trail, k);
    if (t[k] >= uint32_t(V)) atomicMin(&valid_end, k);
  }
  __syncthreads();
  // The leading run began `back` rows earlier: a short one is the previous chunk's.  The trailing
  // run starts at `trail` and ends at trail_end.
  const bool open = back > 0, lead_long = back + lead_end > chunk;
  const bool trail_long = t[trail + chunk] == last;   // trail + chunk < 2 chunk
  int k = open && !lead_long ? lead_end : 0;
  int end = trail_long ? n : trail_end;
  end = min(end, valid_end);
  const int pack = slice * kChunkThreads + tid, packs = d / kCols;
  if (k >= end || pack >= packs) return;
  const Pack<E, kCols>* src = reinterpret_cast<const Pack<E, kCols>*>(dY) + pack;
  float acc[kCols] = {};
  auto flush = [&](int from) {   // the run that began at (or before) `from`
    const bool is_lead = from == 0 && open, is_trail = from == trail && trail_long;
    if (is_lead || is_trail)
      put_sum(part + ((long long)c * 2 + (is_lead ? 0 : 1)) * d + pack * kCols, acc, 1.f, false);
    else
      put_sum(dE + (long long)t[from] * d + pack * kCols, acc, scale, accumulate != 0);
#pragma unroll
    for (int j = 0; j < kCols; ++j) acc[j] = 0.f;
  };
  int from = k;
  for (; k < end; k += kChunkBatch) {
    Pack<E, kCols> x[kChunkBatch];
#pragma unroll
    for (int j = 0; j < kChunkBatch; ++j)
      if (k + j < end) x[j] = src[(long long)row[k + j] * packs];
#pragma unroll
    for (int j = 0; j < kChunkBatch; ++j) {
      if (k + j >= end) break;
      if (t[k + j] != t[from]) {
        flush(from);
        from = k + j;
      }
      add_pack(acc, x[j]);
    }
  }
  flush(from);
}

// --- long runs: partial sums of the chunks, in order.  A warp takes 128 columns of a run; of a run
// of many chunks the block's warps take an equal share each, joined in order through shared memory.
// The items (run, 128 columns) go to the blocks in turn, so that the columns of one run of many
// chunks are different blocks' (in an earlier form, eight to a
// block, the join took 145 us for one run of 480 chunks, 2048 columns).
constexpr int kJoinThreads = 1024;
constexpr int kJoinWarps = kJoinThreads / 32;
constexpr int kJoinFew = 16;   // partial sums that one warp adds

ALR_DEV float4 join_parts(const float* part, int d, int col, int c, int from, int to) {
  // partial sum 0 is the run's start (slot 1 of chunk c), the others slot 0 of the next chunks
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (int k = from; k < to; ++k) {
    const float* p = part + ((long long)(c + k) * 2 + (k == 0 ? 1 : 0)) * d + col;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (d % 4 == 0) {
      x = *reinterpret_cast<const float4*>(p);
    } else {
      x.x = p[0];
      if (col + 1 < d) x.y = p[1];
      if (col + 2 < d) x.z = p[2];
      if (col + 3 < d) x.w = p[3];
    }
    s.x += x.x;
    s.y += x.y;
    s.z += x.z;
    s.w += x.w;
  }
  return s;
}

ALR_DEV void put_join(float* dE, uint32_t t, int d, int col, float4 s, float scale,
                      bool accumulate) {
  const float v[4] = {s.x, s.y, s.z, s.w};
  for (int j = 0; j < 4 && col + j < d; ++j) {
    float* p = dE + (long long)t * d + col + j;
    *p = fmaf(scale, v[j], accumulate ? *p : 0.f);
  }
}

__global__ void __launch_bounds__(kJoinThreads)
    embed_join_kernel(int d, const uint32_t* tok_s, int N, int chunk, const int2* list,
                      const int32_t* count, float scale, int accumulate, const float* part,
                      float* dE) {
  __shared__ float4 sums[kJoinWarps][32];
  __shared__ int4 todo[kJoinWarps];   // chunk, partial sums (0: done), token, column group
  pdl_wait_and_release();
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const int groups = (d + 127) / 128, items = *count * groups;
  for (int i0 = 0; i0 < items; i0 += gridDim.x * kJoinWarps) {
    const int i = i0 + warp * gridDim.x + blockIdx.x;
    if (lane == 0) todo[warp] = make_int4(0, 0, 0, 0);
    if (i < items) {
      const int2 run = list[i / groups];
      const int g = i % groups, c = run.x / chunk;
      const uint32_t t = uint32_t(run.y);
      // chunks after c that begin with the token: lanes test 32 of them, ever closer together
      int more = 0;
      for (int step = N / chunk < 1024 ? 32 : 1 << 15; step > 0; step >>= 5) {
        const long long at = (long long)(c + more + (lane + 1) * (long long)step) * chunk;
        more += step * __popc(__ballot_sync(0xffffffffu, at < N && tok_s[at < N ? at : 0] == t));
      }
      const int n = 1 + more, col = g * 128 + lane * 4;
      if (n > kJoinFew) {
        if (lane == 0) todo[warp] = make_int4(c, n, int(t), g);
      } else if (col < d) {
        put_join(dE, t, d, col, join_parts(part, d, col, c, 0, n), scale, accumulate != 0);
      }
    }
    __syncthreads();
    for (int w = 0; w < kJoinWarps; ++w) {
      const int4 it = todo[w];
      if (it.y == 0) continue;
      const int col = it.w * 128 + lane * 4, share = (it.y + kJoinWarps - 1) / kJoinWarps;
      if (col < d)
        sums[warp][lane] = join_parts(part, d, col, it.x, min(it.y, warp * share),
                                      min(it.y, (warp + 1) * share));
      __syncthreads();
      if (warp == 0 && col < d) {
        float4 s = sums[0][lane];
        for (int k = 1; k < kJoinWarps; ++k) {
          s.x += sums[k][lane].x;
          s.y += sums[k][lane].y;
          s.z += sums[k][lane].z;
          s.w += sums[k][lane].w;
        }
        put_join(dE, uint32_t(it.z), d, col, s, scale, accumulate != 0);
      }
      __syncthreads();
    }
    __syncthreads();
  }
}

template <typename E, int kCols>
cudaError_t embed_grad_cols(const E* dY, int V, int d, const int32_t* tokens, int N, float scale,
                            bool accumulate, float* dE, unsigned char* ws, int sms,
                            cudaStream_t s) {
  const int packs = d / kCols, zero_blocks = accumulate ? 0 : (V + 31) / 32;
  if (N <= kFewRows) {
    // narrow slices, and so many groups for a token of many rows, while the blocks fit the device
    const int lanes = (long long)N * ((packs + 15) / 16) <= 16 * sms ? 16 : 64;
    const int slices = (packs + lanes - 1) / lanes;
    if (N == 0 && accumulate) return cudaSuccess;
    return launch_pdl(embed_grad_few_kernel<E, kCols>, dim3(unsigned(N * slices + zero_blocks)),
                      dim3(kFewThreads), 0, s, dY, V, d, tokens, N, slices, lanes, scale,
                      int(accumulate), dE);
  }
  const GradPlan g = grad_plan(V, d, N);
  uint32_t* tok[2] = {reinterpret_cast<uint32_t*>(ws + g.tok_off[0]),
                      reinterpret_cast<uint32_t*>(ws + g.tok_off[1])};
  uint32_t* row[2] = {reinterpret_cast<uint32_t*>(ws + g.row_off[0]),
                      reinterpret_cast<uint32_t*>(ws + g.row_off[1])};
  int2* list = reinterpret_cast<int2*>(ws + g.list_off);
  int32_t* count = reinterpret_cast<int32_t*>(ws + g.count_off);
  uint32_t* present = accumulate ? nullptr : reinterpret_cast<uint32_t*>(ws + g.present_off);
  float* part = reinterpret_cast<float*>(ws + g.part_off);
  cudaLaunchAttribute attr[2] = {pdl_attribute(), {}};
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kSortCtas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(kSortCtas);
  cfg.blockDim = dim3(kSortThreads);
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  cudaError_t e = cudaLaunchKernelEx(&cfg, embed_sort_kernel, tokens, N, V, g.passes, g.bits,
                                     g.chunk, tok[0], row[0], tok[1], row[1], present, list, count);
  if (e != cudaSuccess) return e;
  const int in = (g.passes - 1) & 1;   // the last pass's output
  const int slices = (packs + kChunkThreads - 1) / kChunkThreads;
  e = launch_pdl(embed_chunk_kernel<E, kCols>, dim3(unsigned(g.n_chunks * slices + zero_blocks)),
                 dim3(kChunkThreads), 0, s, dY, V, d, tok[in], row[in], N, g.chunk, g.n_chunks,
                 slices, scale, int(accumulate), dE, part, present);
  if (e != cudaSuccess) return e;
  return launch_pdl(embed_join_kernel, dim3(unsigned(sms)), dim3(kJoinThreads), 0, s, d, tok[in],
                    N, g.chunk, list, count, scale, int(accumulate), part, dE);
}

}  // namespace

cudaError_t launch_embed(int dtype, const void* table, int V, int d, const int32_t* tokens,
                         long long N, float scale, void* out, cudaStream_t s) {
  auto run = [&](auto kern, int cols, auto* t, auto* o) {
    const int packs = d / cols, pieces = (packs + 32 * kEmbedBatch - 1) / (32 * kEmbedBatch);
    const long long warps = N * pieces, per = kEmbedThreads / 32;
    return launch_pdl(kern, dim3(unsigned((warps + per - 1) / per)), dim3(kEmbedThreads), 0, s, t, V,
                      packs, pieces, tokens, N, scale, o);
  };
  if (dtype == 0) {
    auto* t = static_cast<const __nv_bfloat16*>(table);
    auto* o = static_cast<__nv_bfloat16*>(out);
    return d % 8 == 0   ? run(embed_kernel<__nv_bfloat16, 8>, 8, t, o)
           : d % 2 == 0 ? run(embed_kernel<__nv_bfloat16, 2>, 2, t, o)
                        : run(embed_kernel<__nv_bfloat16, 1>, 1, t, o);
  }
  auto* t = static_cast<const float*>(table);
  auto* o = static_cast<float*>(out);
  return d % 4 == 0 ? run(embed_kernel<float, 4>, 4, t, o) : run(embed_kernel<float, 1>, 1, t, o);
}

cudaError_t launch_embed_grad(int dtype, const void* dY, int V, int d, const int32_t* tokens,
                              int N, float scale, bool accumulate, float* dE, void* workspace,
                              int sms, cudaStream_t s) {
  auto run = [&](auto cols, auto* y) {
    using E = std::remove_cv_t<std::remove_pointer_t<decltype(y)>>;
    return embed_grad_cols<E, decltype(cols)::value>(y, V, d, tokens, N, scale, accumulate, dE,
                                                     static_cast<unsigned char*>(workspace), sms, s);
  };
  if (dtype == 0) {
    auto* y = static_cast<const __nv_bfloat16*>(dY);
    return d % 8 == 0   ? run(std::integral_constant<int, 8>{}, y)
           : d % 2 == 0 ? run(std::integral_constant<int, 2>{}, y)
                        : run(std::integral_constant<int, 1>{}, y);
  }
  auto* y = static_cast<const float*>(dY);
  return d % 4 == 0 ? run(std::integral_constant<int, 4>{}, y)
                    : run(std::integral_constant<int, 1>{}, y);
}

size_t embed_grad_workspace(int V, int d, int N) {
  return N <= kFewRows ? 256 : grad_plan(V, d, N).total;
}

}  // namespace alr
