// Rows of a table by id, scaled, and the gradient of the table.
//
// out[i] = scale * table[ids[i]] is a gather: bytes of the distinct rows and of the output bound it.  The gradient,
// dtable[r] = scale * sum of dout[i] over ids[i] = r, is summed in a fixed order instead of by atomics: ids are sorted with their places
// (least digit first, 8 bits at most at a time, stable, a kernel per digit), and runs of equal ids in the sorted order are summed.  Chunks of that order go to groups of
// lanes; what runs have in neighboring chunks is added up within a thread block, in order, and a run across blocks leaves one partial sum per block, which a
// last kernel adds in order.  Rows that no id names are zeros: the blocks beside the sorting ones write them while the sort, which waits on latency, runs.
// Few ids over few rows are not sorted: the blocks, each with some rows of the table, look through all of them.
#include <type_traits>

#include "tgnn_table.cuh"

using namespace tgnn_table;

namespace {

constexpr int kSortThreads = 1024;
constexpr int kMaxSortBlocks = 148;
constexpr int kDigits = 256;
constexpr int kMaxPasses = 4;

// ------------------------------------------------------------------------------------------------------------ forward --
struct GatherArgs {
  const void* table;
  const void* ids;
  void* out;
  int32_t* status;
  int64_t rows, n;
  float scale;
  int dim, groups;        // groups of V values per row
  int rows_per_block;
  uint32_t magic;         // ceil(2^32 / groups): x * magic >> 32 = x / groups for x * groups < 2^32; 0 for groups = 1
};

template <typename TT, typename TO, int V, typename I>
__global__ void __launch_bounds__(256) lookup_kernel(const GatherArgs a) {
  const int64_t r0 = (int64_t)blockIdx.x * a.rows_per_block;
  const int count = (int)min((int64_t)a.rows_per_block, a.n - r0) * a.groups;
  const I* ids = static_cast<const I*>(a.ids) + r0;
  TO* out = static_cast<TO*>(a.out) + r0 * a.dim;
  const char* const base = static_cast<const char*>(a.table);
  const uint32_t row_bytes = (uint32_t)a.dim * (uint32_t)sizeof(TT);
  typedef typename std::make_unsigned<I>::type Unsigned;
  constexpr int U = 4;
  for (int x0 = threadIdx.x; x0 < count; x0 += 256 * U) {
    uint32_t at[U];                                                            // byte in the row
    I id[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t x = x0 + 256 * u, row = a.magic ? __umulhi(x, a.magic) : x;
      at[u] = (x - row * a.groups) * (V * (uint32_t)sizeof(TT));
      id[u] = x < (uint32_t)count ? ids[row] : (I)-1;
    }
    Group<TT, V> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if ((Unsigned)id[u] < (Unsigned)a.rows) v[u] = *reinterpret_cast<const Group<TT, V>*>(base + (uint64_t)id[u] * row_bytes + at[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = x0 + 256 * u;
      if (x >= count) break;
      float f[V];
      if ((Unsigned)id[u] < (Unsigned)a.rows) {
        v[u].get(f);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] *= a.scale;
      } else {
        if (id[u] >= 0) *a.status = 4;
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = 0.f;
      }
      TO* p = out + (uint32_t)x * V;
      constexpr int W = V * sizeof(TO) > 16 ? 16 / (int)sizeof(TO) : V;        // values per store
#pragma unroll
      for (int i = 0; i < V; i += W) {
        Group<TO, W> g;
        g.set(f + i);
        *reinterpret_cast<Group<TO, W>*>(p + i) = g;
      }
    }
  }
}

// --------------------------------------------------------------------------------------------------------------- sort --
struct SortArgs {
  const void* ids;
  int index_bits;
  int64_t rows;
  uint32_t n;
  const uint2* in;        // (id, place) of the pass before; nullptr: the ids themselves
  uint2* out;
  uint32_t* hist;         // [sort blocks][kDigits]: of this pass
  uint32_t* next_hist;    // of the next one, counted as keys are moved; nullptr: there is none
  int later_words;        // words of those of all later passes, which lie one behind the other: zeroed by the first kernel
  int32_t* status;        // checked on the first look at the ids; nullptr afterwards
  uint32_t* counter;      // zeroed by the first kernel
  int shift, width;       // the digit
  int sort_blocks;
  uint32_t per_block;
  char* zero;             // dtable: blocks behind the sorting ones fill their share of it with zeros
  int64_t zero_bytes;
  int share, shares;
};

// An id as a key: ids below 0 and outside the table come last, as `rows`.
__device__ __forceinline__ uint32_t key_of(const SortArgs& a, uint32_t i) {
  const int64_t id = a.index_bits == 64 ? static_cast<const int64_t*>(a.ids)[i] : static_cast<const int32_t*>(a.ids)[i];
  if (id >= 0 && id < a.rows) return (uint32_t)id;
  if (id >= 0 && a.status) *a.status = 4;
  return (uint32_t)a.rows;
}

__device__ __forceinline__ void fill_zero(const SortArgs& a, int block, int blocks) {
  char* lo = reinterpret_cast<char*>(((uintptr_t)a.zero + 15) & ~(uintptr_t)15);
  char* end = a.zero + a.zero_bytes;
  if (lo > end) lo = end;
  const int64_t words = (end - lo) >> 4;
  const int64_t w0 = words * a.share / a.shares, w1 = words * (a.share + 1) / a.shares;
  for (int64_t w = w0 + (int64_t)block * blockDim.x + threadIdx.x; w < w1; w += (int64_t)blocks * blockDim.x)
    __stcs(reinterpret_cast<uint4*>(lo) + w, make_uint4(0, 0, 0, 0));
  if (a.share == 0 && block == 0 && threadIdx.x == 0) {                       // what lies before and behind whole words, by 2 bytes
    for (char* p = a.zero; p < lo; p += 2) *reinterpret_cast<uint16_t*>(p) = 0;
    for (char* p = lo + 16 * words; p < end; p += 2) *reinterpret_cast<uint16_t*>(p) = 0;
  }
}

// Ranks of a warp's keys among those of the warp with the same digit, in order: lanes, then rounds.  `mine` counts the warp's digits.
template <int K>
__device__ __forceinline__ void rank_keys(const uint32_t (&digit)[K], uint32_t (&rank)[K], uint32_t* mine, int lane) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const unsigned same = __match_any_sync(FULL, digit[k]);
    const int leader = __ffs(same) - 1;
    uint32_t before = 0;
    if (lane == leader && digit[k] < kDigits) {
      before = mine[digit[k]];
      mine[digit[k]] = before + __popc(same);
    }
    before = __shfl_sync(FULL, before, leader);
    rank[k] = before + __popc(same & ((1u << lane) - 1));
    __syncwarp();
  }
}

// counts[warp][digit] -> where that warp's keys of the digit begin within the block, total[digit] = keys of the block.  1024 threads: four
// groups of eight warps, a thread per group and digit.
__device__ __forceinline__ void scan_warps(uint32_t (*counts)[kDigits], uint32_t (*part)[kDigits], uint32_t* total) {
  const int d = threadIdx.x & (kDigits - 1), grp = threadIdx.x >> 8;
  uint32_t c[8], sum = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    c[w] = counts[8 * grp + w][d];
    const uint32_t x = c[w];
    c[w] = sum;
    sum += x;
  }
  part[grp][d] = sum;
  __syncthreads();
  uint32_t at = 0;
  for (int g = 0; g < grp; ++g) at += part[g][d];
  if (grp == 3) total[d] = at + sum;
#pragma unroll
  for (int w = 0; w < 8; ++w) counts[8 * grp + w][d] = c[w] + at;
  __syncthreads();
}

// Exclusive sums of total[] into base[], by the first eight warps.
__device__ __forceinline__ void scan_digits(const uint32_t* total, uint32_t* base, uint32_t* warp_sum) {
  const int t = threadIdx.x, lane = t & 31;
  uint32_t x = 0, inc = 0;
  if (t < kDigits) {
    x = inc = total[t];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(FULL, inc, o);
      if (lane >= o) inc += y;
    }
    if (lane == 31) warp_sum[t >> 5] = inc;
  }
  __syncthreads();
  if (t < kDigits) {
    uint32_t at = inc - x;
    for (int w = 0; w < (t >> 5); ++w) at += warp_sum[w];
    base[t] = at;
  }
  __syncthreads();
}

// A kernel counts the first digits of every block's share, and one per digit moves the keys and counts the next digits where they come to lie.
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const SortArgs a) {
  __shared__ uint32_t count[kDigits];
  chain_wait();
  chain_release();
  if ((int)blockIdx.x >= a.sort_blocks) {
    fill_zero(a, blockIdx.x - a.sort_blocks, gridDim.x - a.sort_blocks);
    return;
  }
  const uint32_t lo = blockIdx.x * a.per_block, hi = min(a.n, lo + a.per_block);
  const uint32_t mask = (1u << a.width) - 1;
  if (threadIdx.x < kDigits) count[threadIdx.x] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.counter = 0;
  for (int i = blockIdx.x * kSortThreads + threadIdx.x; i < a.later_words; i += a.sort_blocks * kSortThreads) a.next_hist[i] = 0;
  __syncthreads();
  constexpr int K = 4;
  for (uint32_t tile = lo; tile < hi; tile += K * kSortThreads) {
    uint32_t d[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t i = tile + k * kSortThreads + threadIdx.x;
      d[k] = i < hi ? key_of(a, i) & mask : kDigits;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const unsigned same = __match_any_sync(FULL, d[k]);                     // hubs: one addition per warp and digit
      if ((threadIdx.x & 31) == __ffs(same) - 1 && d[k] < kDigits) atomicAdd(count + d[k], __popc(same));
    }
  }
  __syncthreads();
  if (threadIdx.x < kDigits) a.hist[blockIdx.x * kDigits + threadIdx.x] = count[threadIdx.x];
}

template <int K>
__global__ void __launch_bounds__(kSortThreads) sort_move_kernel(const SortArgs a) {
  __shared__ uint32_t counts[32][kDigits];
  __shared__ uint32_t part[4][kDigits], total[kDigits], base[kDigits], warp_sum[8];
  chain_wait();
  chain_release();
  if ((int)blockIdx.x >= a.sort_blocks) {
    fill_zero(a, blockIdx.x - a.sort_blocks, gridDim.x - a.sort_blocks);
    return;
  }
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  {  // where this block's keys of every digit begin: all keys of smaller digits, and the blocks before it
    const int d = t & (kDigits - 1), grp = t >> 8, me = blockIdx.x;
    const int b0 = a.sort_blocks * grp / 4, b1 = a.sort_blocks * (grp + 1) / 4;
    uint32_t all = 0, before = 0;
#pragma unroll 8
    for (int b = b0; b < b1; ++b) {
      const uint32_t x = a.hist[b * kDigits + d];
      all += x;
      before += b < me ? x : 0;
    }
    part[grp][d] = all;
    counts[grp][d] = before;
    __syncthreads();
    if (t < kDigits) total[t] = part[0][t] + part[1][t] + part[2][t] + part[3][t];
    __syncthreads();
    scan_digits(total, base, warp_sum);
    if (t < kDigits) base[t] += counts[0][t] + counts[1][t] + counts[2][t] + counts[3][t];
    __syncthreads();
  }
  const uint32_t lo = blockIdx.x * a.per_block, hi = min(a.n, lo + a.per_block);
  const uint32_t mask = (1u << a.width) - 1;
  for (uint32_t tile = lo; tile < hi; tile += K * kSortThreads) {
    for (int i = t; i < 32 * kDigits; i += kSortThreads) (&counts[0][0])[i] = 0;
    __syncthreads();
    uint2 kp[K];
    uint32_t digit[K], rank[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t i = tile + warp * (32 * K) + 32 * k + lane;
      digit[k] = kDigits;
      if (i < hi) {
        kp[k] = a.in ? a.in[i] : make_uint2(key_of(a, i), i);
        digit[k] = (kp[k].x >> a.shift) & mask;
      }
    }
    rank_keys<K>(digit, rank, counts[warp], lane);
    __syncthreads();
    scan_warps(counts, part, total);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      uint32_t counted = 0xffffffffu;
      if (digit[k] < kDigits) {
        const uint32_t to = base[digit[k]] + counts[warp][digit[k]] + rank[k];
        a.out[to] = kp[k];
        if (a.next_hist) counted = to / a.per_block * kDigits + ((kp[k].x >> (a.shift + a.width)) & mask);
      }
      if (a.next_hist) {                                                       // whole numbers: the order of additions does not matter
        const unsigned same = __match_any_sync(FULL, counted);
        if (lane == __ffs(same) - 1 && counted != 0xffffffffu) atomicAdd(a.next_hist + counted, __popc(same));
      }
    }
    __syncthreads();
    if (t < kDigits) base[t] += total[t];
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------------------- run sums --
struct SumArgs {
  const uint2* sorted;
  const void* dout;
  void* dtable;
  int dtype;              // of dtable
  float* partial;         // [block][head, tail][dim]
  uint8_t* through;       // [block]: the run at its start goes on behind its end
  uint32_t* list;         // blocks at whose end a run that begins in them goes on
  uint32_t* counter;
  uint32_t n, rows;
  int dim, groups, chunk, span;   // span: ids of a thread block
  float scale;
};

__device__ __forceinline__ void store_row(void* base, int dtype, int64_t at, float x) {
  if (dtype == TGNN_F32) static_cast<float*>(base)[at] = x;
  else if (dtype == TGNN_BF16) static_cast<__nv_bfloat16*>(base)[at] = __float2bfloat16_rn(x);
  else static_cast<__half*>(base)[at] = __float2half_rn(x);
}
template <int V>
__device__ __forceinline__ void store_values(void* base, int dtype, int64_t at, const float* x) {
  if (dtype == TGNN_F32) {
    constexpr int W = V > 4 ? 4 : V;
#pragma unroll
    for (int i = 0; i < V; i += W) {
      Group<float, W> g;
      g.set(x + i);
      if (V == 1 || (((uintptr_t)base & (4 * W - 1)) == 0)) *reinterpret_cast<Group<float, W>*>(static_cast<float*>(base) + at + i) = g;
      else
        for (int j = 0; j < W; ++j) static_cast<float*>(base)[at + i + j] = x[i + j];
    }
  } else {
    const bool wide = ((uintptr_t)base & (2 * V - 1)) == 0;
    if (wide) {
      if (dtype == TGNN_BF16) {
        Group<__nv_bfloat16, V> g;
        g.set(x);
        *reinterpret_cast<Group<__nv_bfloat16, V>*>(static_cast<__nv_bfloat16*>(base) + at) = g;
      } else {
        Group<__half, V> g;
        g.set(x);
        *reinterpret_cast<Group<__half, V>*>(static_cast<__half*>(base) + at) = g;
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) store_row(base, dtype, at + i, x[i]);
    }
  }
}

// G lanes take a chunk of the sorted order and V values each of a slice of G * V columns (grid.y slices).  Eight rows are asked for before
// the first is added, and the ids of the next eight.
template <typename T, int V, int G>
__global__ void __launch_bounds__(256) run_sum_kernel(const SumArgs a) {
  constexpr int NG = 256 / G;
  __shared__ float s_head[NG][G * V];
  __shared__ uint8_t s_through[NG];
  chain_wait();
  chain_release();
  const int lane = threadIdx.x & (G - 1), grp = threadIdx.x / G;
  const int col = blockIdx.y * G + lane;
  const int64_t t0 = min((int64_t)a.n, ((int64_t)blockIdx.x * NG + grp) * a.chunk);
  const uint32_t end = (uint32_t)min((int64_t)a.n, t0 + a.chunk);
  const bool active = col < a.groups;
  const T* dout = static_cast<const T*>(a.dout) + col * V;
  uint32_t cur = t0 < end ? a.sorted[t0].x : 0xffffffffu;
  const bool head = t0 > 0 && cur < a.rows && a.sorted[t0 - 1].x == cur;      // the first run began in an earlier chunk
  bool whole = true;                                                          // no run has ended yet
  float acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.f;
  constexpr int U = 8;
  auto write = [&]() {
    if (!active) return;
    float x[V];
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = acc[i] * a.scale;
    store_values<V>(a.dtable, a.dtype, (int64_t)cur * a.dim + col * V, x);
  };
  auto keep = [&]() {                                                         // what the first run has here
#pragma unroll
    for (int i = 0; i < V; ++i) s_head[grp][lane * V + i] = acc[i];
  };
  uint2 next[U];
#pragma unroll
  for (int u = 0; u < U; ++u) next[u] = t0 + u < end ? a.sorted[t0 + u] : make_uint2(0xffffffffu, 0);
  for (uint32_t t = (uint32_t)t0; t < end && cur < a.rows; t += U) {
    uint2 kp[U];
    Group<T, V> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      kp[u] = next[u];
      next[u] = t + U + u < end ? a.sorted[t + U + u] : make_uint2(0xffffffffu, 0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (active && kp[u].x < a.rows) v[u] = *reinterpret_cast<const Group<T, V>*>(dout + (int64_t)kp[u].y * a.dim);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t + u >= end) break;
      if (kp[u].x != cur) {
        if (head && whole) keep();
        else write();
        whole = false;
        cur = kp[u].x;
        if (cur >= a.rows) break;
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = 0.f;
      }
      float f[V];
      v[u].get(f);
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] += f[i];
    }
  }
  const bool goes_on = cur < a.rows && end < a.n && a.sorted[end].x == cur, begun = head && whole && cur < a.rows;
  if (begun) keep();
  else if (cur < a.rows && !goes_on) write();
  if (lane == 0) s_through[grp] = begun && goes_on;
  __syncthreads();
  // Runs across the block's chunks: the group that a run begins in adds what the next ones have of it; the first group does so for the run that the
  // block before began.
  auto follow = [&](int g) {                                                  // from group g on; whether the run goes on behind the block
    for (; g < NG; ++g) {
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] += s_head[g][lane * V + i];
      if (!s_through[g]) return false;
    }
    return true;
  };
  auto part = [&](int slot) {
    if (!active) return;
    float* p = a.partial + ((int64_t)2 * blockIdx.x + slot) * a.dim + col * V;
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = acc[i];
  };
  if (goes_on && !begun) {
    if (follow(grp + 1)) {
      part(1);
      if (lane == 0 && blockIdx.y == 0) a.list[atomicAdd(a.counter, 1u)] = blockIdx.x;
    } else {
      write();
    }
  }
  if (grp == 0) {
    bool on = false;
    if (head) {
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] = 0.f;
      on = follow(0);
      part(0);
    }
    if (lane == 0 && blockIdx.y == 0) a.through[blockIdx.x] = on;
  }
}

// Few ids and few rows: a thread block per `kRows` rows of the table and slice of 32 * V columns looks through all ids, every warp an equal part of them, adds
// up what it finds of its rows in shared memory, in order, and the parts of the warps are added in order.  One kernel in place of a sort's three or four and the sums' two.  The rows of
// a block are as far apart as there are blocks: hubs often have neighboring numbers.
struct FewArgs {
  const void* ids;
  const void* dout;
  void* dtable;
  int32_t* status;
  int64_t rows;
  int index_bits, n, dim, dtype;
  uint32_t magic;         // ceil(2^32 / blocks of rows), 0 for one block: x * magic >> 32 = x / blocks for x * blocks < 2^32
  float scale;
};
constexpr int kFewWarps = 16;
template <typename T, int V>
__global__ void __launch_bounds__(32 * kFewWarps) few_sum_kernel(const FewArgs a) {
  constexpr int kRows = 32 / V, kHeld = 128;
  extern __shared__ float s_sum[];                                            // [warp][row][V][32]
  __shared__ uint16_t s_place[kFewWarps][kHeld];
  __shared__ uint8_t s_row[kFewWarps][kHeld];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int col = (blockIdx.y * 32 + lane) * V;
  const bool active = col < a.dim;
  const T* dout = static_cast<const T*>(a.dout) + col;
  float* mine = s_sum + warp * kRows * 32 * V + lane;
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int k = 0; k < V; ++k) mine[(r * V + k) * 32] = 0.f;
  const int per = (a.n + kFewWarps - 1) / kFewWarps, lo = min(a.n, warp * per), hi = min(a.n, lo + per);
  int held = 0;
  auto flush = [&]() {
    __syncwarp();
    for (int u0 = 0; u0 < held; u0 += 8) {
      Group<T, V> v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (u0 + u < held && active) v[u] = *reinterpret_cast<const Group<T, V>*>(dout + (int64_t)s_place[warp][u0 + u] * a.dim);
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (u0 + u < held) {
          float f[V], *x = mine + s_row[warp][u0 + u] * 32 * V;
          v[u].get(f);
#pragma unroll
          for (int k = 0; k < V; ++k) x[32 * k] += f[k];
        }
    }
    held = 0;
    __syncwarp();
  };
  bool beyond = false;
  for (int j0 = lo; j0 < hi; j0 += 128) {
    int64_t id[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int j = j0 + 32 * k + lane;
      id[k] = -1;
      if (j < hi) id[k] = a.index_bits == 64 ? static_cast<const int64_t*>(a.ids)[j] : (int64_t) static_cast<const int32_t*>(a.ids)[j];
      beyond |= id[k] >= a.rows;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t row = a.magic ? __umulhi((uint32_t)id[k], a.magic) : (uint32_t)id[k];
      const bool here = id[k] >= 0 && id[k] < a.rows && (uint32_t)id[k] - row * gridDim.x == blockIdx.x;
      const unsigned hits = __ballot_sync(FULL, here);
      if (hits == 0) continue;
      if (held + __popc(hits) > kHeld) flush();
      if (here) {
        const int at = held + __popc(hits & ((1u << lane) - 1));
        s_place[warp][at] = (uint16_t)(j0 + 32 * k + lane);
        s_row[warp][at] = (uint8_t)row;
      }
      held += __popc(hits);
    }
  }
  flush();
  if (beyond) *a.status = 4;
  __syncthreads();
  for (int r = warp; r < kRows; r += kFewWarps) {
    const int64_t row = (int64_t)r * gridDim.x + blockIdx.x;
    if (row >= a.rows) break;
    float x[V];
#pragma unroll
    for (int k = 0; k < V; ++k) x[k] = 0.f;
    for (int w = 0; w < kFewWarps; ++w)
#pragma unroll
      for (int k = 0; k < V; ++k) x[k] += s_sum[((w * kRows + r) * V + k) * 32 + lane];
#pragma unroll
    for (int k = 0; k < V; ++k) x[k] *= a.scale;
    if (active) store_values<V>(a.dtable, a.dtype, row * a.dim + col, x);
  }
}

// Runs across blocks: tail of the block that they begin in, then the heads of the next ones.  A warp per run of up to 16 heads; longer ones (hubs) are put
// aside and taken by the whole block, every warp its part of the heads.  The list's order does not matter.
constexpr int kJoinWarps = 16, kAside = 256;
template <int V>
__device__ __forceinline__ void add_part(const float* p, float* x) {
  float f[V];
  reinterpret_cast<const Group<float, V>*>(p)->get(f);
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] += f[i];
}
template <int V>
__global__ void __launch_bounds__(32 * kJoinWarps) run_join_kernel(const SumArgs a, uint32_t chunks) {
  chain_wait();
  chain_release();
  __shared__ float sum[kJoinWarps][32 * V];
  __shared__ uint32_t aside[kAside], s_count, s_last;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t runs = *a.counter;
  const int col = (blockIdx.y * 32 + lane) * V;
  const bool active = col < a.dim;
  if (threadIdx.x == 0) s_count = 0;
  __syncthreads();
  auto finish = [&](uint32_t c0, float* x) {
    if (!active) return;
    const uint32_t id = a.sorted[(int64_t)(c0 + 1) * a.span].x;
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] *= a.scale;
    store_values<V>(a.dtable, a.dtype, (int64_t)id * a.dim + col, x);
  };
  for (uint32_t r = blockIdx.x * kJoinWarps + warp; r < runs; r += gridDim.x * kJoinWarps) {
    const uint32_t c0 = a.list[r], c = c0 + 1 + lane;
    const unsigned ends = __ballot_sync(FULL, c >= chunks || !a.through[c]) & 0xffffu;
    if (ends == 0) {                                                           // more than 16 heads
      uint32_t at = 0;
      if (lane == 0) at = atomicAdd(&s_count, 1u);
      at = __shfl_sync(FULL, at, 0);
      if (at < kAside) {
        if (lane == 0) aside[at] = c0;
        continue;
      }
    }
    uint32_t heads = __ffs(ends);
    float x[V];
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = 0.f;
    if (ends == 0) {                                                           // there was no room to put it aside: the same sums in the same order
      for (heads = 17; c0 + heads < chunks && a.through[c0 + heads]; ++heads) {}
      for (int w = 0; w < kJoinWarps && active; ++w) {
        float y[V];
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = 0.f;
        if (w == 0) add_part<V>(a.partial + ((int64_t)2 * c0 + 1) * a.dim + col, y);
        for (uint32_t h = 1 + w; h <= heads && c0 + h < chunks; h += kJoinWarps) add_part<V>(a.partial + (int64_t)2 * (c0 + h) * a.dim + col, y);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = w ? x[i] + y[i] : y[i];
      }
    } else if (active) {
      add_part<V>(a.partial + ((int64_t)2 * c0 + 1) * a.dim + col, x);
#pragma unroll 8
      for (uint32_t h = 1; h <= heads; ++h) add_part<V>(a.partial + (int64_t)2 * (c0 + h) * a.dim + col, x);
    }
    finish(c0, x);
  }
  __syncthreads();
  const uint32_t long_runs = min(s_count, (uint32_t)kAside);
  for (uint32_t r = 0; r < long_runs; ++r) {
    const uint32_t c0 = aside[r];
    uint32_t last = c0 + 1;                                                    // the last chunk that the run reaches
    for (;; last += 32 * kJoinWarps) {
      if (threadIdx.x == 0) s_last = 0xffffffffu;
      __syncthreads();
      const uint32_t c = last + threadIdx.x;
      if (c >= chunks || !a.through[c]) atomicMin(&s_last, c);
      __syncthreads();
      const uint32_t x = s_last;
      __syncthreads();
      if (x != 0xffffffffu) {
        last = min(x, chunks - 1);
        break;
      }
    }
    float x[V];
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = 0.f;
    if (active) {
      if (warp == 0) add_part<V>(a.partial + ((int64_t)2 * c0 + 1) * a.dim + col, x);
#pragma unroll 8
      for (uint32_t c = c0 + 1 + warp; c <= last; c += kJoinWarps) add_part<V>(a.partial + (int64_t)2 * c * a.dim + col, x);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) sum[warp][lane * V + i] = x[i];
    __syncthreads();
    if (warp == 0) {
      for (int w = 1; w < kJoinWarps; ++w)
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] += sum[w][lane * V + i];
      finish(c0, x);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------------------- host side --
template <typename TT, typename TO, int V>
void gather(Chain& c, const GatherArgs& a, int bits, unsigned blocks) {
  if (bits == 64) c(lookup_kernel<TT, TO, V, int64_t>, dim3(blocks), dim3(256), 0, a);
  else c(lookup_kernel<TT, TO, V, int32_t>, dim3(blocks), dim3(256), 0, a);
}
template <typename TT, typename TO>
void gather_type(Chain& c, GatherArgs a, int bits) {
  // the widest group of values that divides a row and that both sides' addresses allow
  constexpr int W = 16 / (int)sizeof(TT);
  auto fits = [&](int v) {
    const int wo = v * (int)sizeof(TO) > 16 ? 16 : v * (int)sizeof(TO);
    return a.dim % v == 0 && ((uintptr_t)a.table & (v * sizeof(TT) - 1)) == 0 && ((uintptr_t)a.out & (wo - 1)) == 0;
  };
  const int v = fits(W) ? W : fits(2) ? 2 : 1;
  a.groups = a.dim / v;
  a.magic = a.groups == 1 ? 0 : (uint32_t)(((1ull << 32) + a.groups - 1) / a.groups);
  a.rows_per_block = a.groups >= 1024 ? 1 : 1024 / a.groups;
  // few rows: fewer per block, so that they reach every multiprocessor
  while (a.rows_per_block > 1 && (int64_t)a.rows_per_block * 2 * num_sms() > a.n && a.rows_per_block * a.groups > 256) a.rows_per_block /= 2;
  const unsigned blocks = (unsigned)((a.n + a.rows_per_block - 1) / a.rows_per_block);
  if (v == W) gather<TT, TO, W>(c, a, bits, blocks);
  else if (v == 2) gather<TT, TO, 2>(c, a, bits, blocks);
  else gather<TT, TO, 1>(c, a, bits, blocks);
}
template <typename TT>
void gather_out(Chain& c, const GatherArgs& a, int out_dtype, int bits) {
  if (out_dtype == TGNN_F32) gather_type<TT, float>(c, a, bits);
  else if (out_dtype == TGNN_BF16) gather_type<TT, __nv_bfloat16>(c, a, bits);
  else gather_type<TT, __half>(c, a, bits);
}

// Ids per group of lanes, with `groups` of them in a thread block: few enough that the groups fill the device, and 1024 or more in a block where there are
// many, so that hubs leave few parts (rows of 100 fp32, 8 groups, chunks of 16 / 32 / 64 / 128 in us, ids of 17 000 nodes drawn with weights 1 / i^1.2:
// 2^16 ids 34 / 36 / 38 / 46, 2^17 58 / 44 / 47 / 59, 2^18 110 / 84 / 70 / 69, 2^20 326 / 249 / 209 / 186, 2^22 1144 / 830 / 676 / 605; drawn evenly
// 2^16 33 / 33 / 38 / 45, 2^20 174 / 170 / 167 / 172).
int chunk_of(int64_t n, int groups) { return n <= 1 << 16 ? 16 : n <= 1 << 17 ? 32 : n <= 1 << 19 || groups > 8 ? 64 : 128; }

template <typename T, int V>
uint32_t sum_lanes(Chain& c, SumArgs& a) {
  uint32_t blocks = 0;
  auto go = [&](auto kernel, int g) {
    a.chunk = chunk_of(a.n, 256 / g);
    a.span = 256 / g * a.chunk;
    blocks = (uint32_t)(((int64_t)a.n + a.span - 1) / a.span);
    c(kernel, dim3(blocks, (a.groups + g - 1) / g), dim3(256), 0, a);
  };
  if (a.groups <= 8) go(run_sum_kernel<T, V, 8>, 8);
  else if (a.groups <= 16) go(run_sum_kernel<T, V, 16>, 16);
  else go(run_sum_kernel<T, V, 32>, 32);
  return blocks;
}
// The widest group of values that divides a row and that the gradient's address allows.
template <typename T>
int width_of(const void* dout, int dim) {
  constexpr int W = 16 / (int)sizeof(T);
  auto fits = [&](int v) { return dim % v == 0 && ((uintptr_t)dout & (v * sizeof(T) - 1)) == 0; };
  return fits(W) ? W : fits(2) ? 2 : 1;
}
template <typename T>
uint32_t sum_type(Chain& c, SumArgs& a) {
  constexpr int W = 16 / (int)sizeof(T);
  const int v = width_of<T>(a.dout, a.dim);
  a.groups = a.dim / v;
  return v == W ? sum_lanes<T, W>(c, a) : v == 2 ? sum_lanes<T, 2>(c, a) : sum_lanes<T, 1>(c, a);
}
template <typename T>
void few_type(Chain& c, const FewArgs& a) {
  constexpr int W = 16 / (int)sizeof(T);
  const int v = width_of<T>(a.dout, a.dim);
  constexpr int kSmem = kFewWarps * 32 * 32 * 4;                               // 32 / v rows of 32 v columns per warp
  auto go = [&](auto kernel) {
    c.e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    const unsigned blocks = (unsigned)((a.rows * v + 31) / 32);
    FewArgs f = a;
    f.magic = blocks == 1 ? 0 : (uint32_t)(((1ull << 32) + blocks - 1) / blocks);
    c(kernel, dim3(blocks, (a.dim + 32 * v - 1) / (32 * v)), dim3(32 * kFewWarps), kSmem, f);
  };
  if (v == W) go(few_sum_kernel<T, W>);
  else if (v == 2) go(few_sum_kernel<T, 2>);
  else go(few_sum_kernel<T, 1>);
}

// Whether every block of rows looks through all ids, or the ids are sorted.  Rows of 100 fp32, us looked through and sorted:
//   ids of nodes       600 of 1000  600 of 16 384  2048 of 9000  2048 of 16 384  6000 of 9000  6000 of 16 384  8192 of 1000  16 384 of 1000
//   drawn evenly        3 and 17      16 and 17      11 and 21     18 and 21       17 and 22     28 and 22        6 and 20     10 and 22
//   weights 1 / i^1.2   4 and 16      15 and 17      10 and 18     16 and 18       18 and 21     26 and 20       23 and 21     49 and 24
//   all one node        8 and 15      14 and 16      21 and 18     23 and 19       60 and 17     62 and 18       81 and 18    161 and 21
bool few(int64_t n, int64_t rows) { return n <= 8192 && rows > 0 && rows <= 16384 && n * rows <= 1 << 26; }

struct Scratch {
  int64_t sorted[2], hist, through, list, counter, partial, bytes;
};
Scratch layout(int64_t n, int dim) {
  const int64_t span = 8 * chunk_of(n, 8), blocks = (n + span - 1) / span;    // of a thread block, at least (8 to 32 groups)
  Scratch s;
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t p = at;
    at += up(bytes, 256);
    return p;
  };
  s.sorted[0] = take(8 * n);
  s.sorted[1] = take(8 * n);
  s.hist = take(4ll * kMaxPasses * kMaxSortBlocks * kDigits);
  s.through = take(blocks);
  s.list = take(4 * blocks);
  s.counter = take(4);
  s.partial = take(8ll * blocks * dim);
  s.bytes = at;
  return s;
}

int check(const char* who, int64_t rows, int dim, int index_bits, int64_t n, int dtype, int out_dtype, char* err, int64_t size) {
  if (!known_dtype(dtype) || !known_dtype(out_dtype)) return fail(err, size, TGNN_EINVAL, "%s: unknown dtype", who);
  if (index_bits != 32 && index_bits != 64) return fail(err, size, TGNN_EINVAL, "%s: index_bits is 32 or 64", who);
  if (rows < 0 || n < 0 || dim < 1 || dim > 8192) return fail(err, size, TGNN_EINVAL, "%s: size out of range (dim 1 to 8192)", who);
  if (rows >= 0x7fffffff || n >= 0x7fffffff) return fail(err, size, TGNN_ECAPACITY, "%s: rows or n beyond int32", who);
  return TGNN_OK;
}

}  // namespace

extern "C" TGNN_API int tgnn_lookup(const void* table, int dtype, int64_t rows, int dim, const void* ids, int index_bits, int64_t n, float scale,
                                    void* out, int out_dtype, int32_t* status, void* stream, char* err, int64_t err_size) {
  const char* who = "tgnn_lookup";
  if (int rc = check(who, rows, dim, index_bits, n, dtype, out_dtype, err, err_size)) return rc;
  if (n == 0) return TGNN_OK;
  if ((rows > 0 && !table) || !ids || !out || !status) return fail(err, err_size, TGNN_EINVAL, "%s: null pointer", who);
  if (((uintptr_t)table & (elem_bytes(dtype) - 1)) || ((uintptr_t)out & (elem_bytes(out_dtype) - 1)) || ((uintptr_t)ids & (index_bits / 8 - 1)) ||
      ((uintptr_t)status & 3))
    return fail(err, err_size, TGNN_EINVAL, "%s: a pointer is not aligned to its element", who);
  GatherArgs a = {};
  a.table = table;
  a.ids = ids;
  a.out = out;
  a.status = status;
  a.rows = rows;
  a.n = n;
  a.scale = scale;
  a.dim = dim;
  Chain c(stream);
  if (dtype == TGNN_F32) gather_out<float>(c, a, out_dtype, index_bits);
  else if (dtype == TGNN_BF16) gather_out<__nv_bfloat16>(c, a, out_dtype, index_bits);
  else gather_out<__half>(c, a, out_dtype, index_bits);
  return c.end(who, err, err_size);
}

extern "C" TGNN_API int64_t tgnn_lookup_scratch(int64_t n, int64_t rows, int dim) {
  if (n < 0 || rows < 0 || n >= 0x7fffffff || rows >= 0x7fffffff || dim < 1 || dim > 8192) return -1;
  return few(n, rows) ? 0 : layout(n, dim).bytes;
}

extern "C" TGNN_API int tgnn_lookup_backward(const void* ids, int index_bits, int64_t n, const void* dout, int out_dtype, int64_t rows, int dim,
                                             float scale, void* dtable, int dtype, void* scratch, int32_t* status, void* stream, char* err,
                                             int64_t err_size) {
  const char* who = "tgnn_lookup_backward";
  if (int rc = check(who, rows, dim, index_bits, n, dtype, out_dtype, err, err_size)) return rc;
  if ((rows > 0 && !dtable) || (n > 0 && (!ids || !dout || !status || (!scratch && !few(n, rows))))) return fail(err, err_size, TGNN_EINVAL, "%s: null pointer", who);
  if (((uintptr_t)dtable & (elem_bytes(dtype) - 1)) || ((uintptr_t)dout & (elem_bytes(out_dtype) - 1)) ||
      ((uintptr_t)ids & (index_bits / 8 - 1)) || ((uintptr_t)scratch & 255) || ((uintptr_t)status & 3))
    return fail(err, err_size, TGNN_EINVAL, "%s: a pointer is not aligned (scratch to 256 bytes, the others to their elements)", who);
  const int64_t bytes = rows * dim * elem_bytes(dtype);
  if (n == 0) {
    if (bytes > 0 && cudaMemsetAsync(dtable, 0, (size_t)bytes, (cudaStream_t)stream) != cudaSuccess)
      return fail(err, err_size, TGNN_ECUDA, "%s: %s", who, cudaGetErrorString(cudaGetLastError()));
    return TGNN_OK;
  }
  SortArgs s = {};
  s.ids = ids;
  s.index_bits = index_bits;
  s.rows = rows;
  s.n = (uint32_t)n;
  s.zero = static_cast<char*>(dtable);
  s.zero_bytes = bytes;
  const int sms = num_sms();
  const int fillers = (int)(bytes >> 14 >= 4 * sms ? 4 * sms : (bytes >> 14) + 1);
  Chain c(stream);
  if (few(n, rows)) {
    FewArgs f = {};
    f.ids = ids;
    f.dout = dout;
    f.dtable = dtable;
    f.status = status;
    f.rows = rows;
    f.index_bits = index_bits;
    f.n = (int)n;
    f.dim = dim;
    f.dtype = dtype;
    f.scale = scale;
    if (out_dtype == TGNN_F32) few_type<float>(c, f);
    else if (out_dtype == TGNN_BF16) few_type<__nv_bfloat16>(c, f);
    else few_type<__half>(c, f);
    return c.end(who, err, err_size);
  }
  const Scratch l = layout(n, dim);
  char* base = static_cast<char*>(scratch);
  int key_bits = 1;
  while ((rows >> key_bits) != 0) ++key_bits;
  s.hist = reinterpret_cast<uint32_t*>(base + l.hist);
  s.status = status;
  s.counter = reinterpret_cast<uint32_t*>(base + l.counter);
  const int passes = (key_bits + 7) / 8;
  s.width = (key_bits + passes - 1) / passes;
  const int64_t tiles = (n + kSortThreads - 1) / kSortThreads;                 // few ids: a key per thread, so that a block's work is short
  s.sort_blocks = (int)(tiles < kMaxSortBlocks ? tiles : kMaxSortBlocks);
  s.per_block = (uint32_t)((n + s.sort_blocks - 1) / s.sort_blocks);
  s.shares = passes + 1;
  const int words = s.sort_blocks * kDigits;
  s.later_words = (passes - 1) * words;
  int sorted = 0;
  for (int p = 0; p < passes; ++p) {
    s.shift = p * s.width;
    s.in = p ? reinterpret_cast<uint2*>(base + l.sorted[sorted]) : nullptr;
    sorted = p & 1;
    s.out = reinterpret_cast<uint2*>(base + l.sorted[sorted]);
    const dim3 grid(s.sort_blocks + fillers), block(kSortThreads);
    if (p == 0) {
      s.share = 0;
      s.next_hist = s.hist + words;
      c(sort_count_kernel, grid, block, 0, s);
      s.status = nullptr;
    } else {
      s.hist += words;
    }
    s.next_hist = p + 1 < passes ? s.hist + words : nullptr;
    s.share = p + 1;
    if (s.per_block <= 1024) c(sort_move_kernel<1>, grid, block, 0, s);
    else if (s.per_block <= 2048) c(sort_move_kernel<2>, grid, block, 0, s);
    else if (s.per_block <= 4096) c(sort_move_kernel<4>, grid, block, 0, s);
    else c(sort_move_kernel<8>, grid, block, 0, s);
  }
  SumArgs a = {};
  a.sorted = reinterpret_cast<uint2*>(base + l.sorted[sorted]);
  a.dout = dout;
  a.dtable = dtable;
  a.dtype = dtype;
  a.partial = reinterpret_cast<float*>(base + l.partial);
  a.through = reinterpret_cast<uint8_t*>(base + l.through);
  a.list = reinterpret_cast<uint32_t*>(base + l.list);
  a.counter = s.counter;
  a.n = (uint32_t)n;
  a.rows = (uint32_t)rows;
  a.dim = dim;
  a.scale = scale;
  const uint32_t blocks = out_dtype == TGNN_F32 ? sum_type<float>(c, a) : out_dtype == TGNN_BF16 ? sum_type<__nv_bfloat16>(c, a) : sum_type<__half>(c, a);
  if (blocks > 1) {
    // four columns per lane where rows allow it; a run per warp at most while the device has room, so that no block is left with many hubs
    const int v = dim % 4 == 0 ? 4 : dim % 2 == 0 ? 2 : 1;
    const unsigned y = (unsigned)(dim + 32 * v - 1) / (32 * v), most = (unsigned)(4 * sms), want = (blocks + kJoinWarps - 1) / kJoinWarps;
    const dim3 grid(want < most ? want : most, y), block(32 * kJoinWarps);
    if (v == 4) c(run_join_kernel<4>, grid, block, 0, a, blocks);
    else if (v == 2) c(run_join_kernel<2>, grid, block, 0, a, blocks);
    else c(run_join_kernel<1>, grid, block, 0, a, blocks);
  }
  return c.end(who, err, err_size);
}
