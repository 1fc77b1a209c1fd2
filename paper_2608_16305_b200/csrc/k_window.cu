// Sampling of a history with a window and sinks: for every root the place of its node's first entry, the number of entries
// strictly earlier than the root's time, and (where asked for) the slots: the most recent `window` of them, then the first
// `sinks` of what the window leaves out.
//
// A warp takes two roots side by side, so that the dependent loads of one (node, slice, search, slots) wait together with the other's.
// The lower bound is found by a 32-way search, as for the most-recent-k search: the lanes probe 32 spread positions with
// independent loads and a ballot picks the sub-range, so a slice of 2*10^7 entries costs 5 dependent loads.  The slots of the window
// lie side by side in the T-CSR; the lanes copy 32 of them at a time.  Small batches are bound by the chain of dependent loads, large
// ones by the slots' bytes.
#include "tgnn_history.cuh"

using namespace tgnn_history;

namespace {

__global__ void __launch_bounds__(128) sample_window_kernel(const int64_t* __restrict__ indptr, const int32_t* __restrict__ g_nbr,
                                                            const int32_t* __restrict__ g_eid, const double* __restrict__ g_ts,
                                                            int64_t N, int64_t P, const int32_t* __restrict__ nodes,
                                                            const double* __restrict__ times, int n, int window, int sinks,
                                                            int32_t* __restrict__ nbr_out, int32_t* __restrict__ eid_out,
                                                            double* __restrict__ ts_out, int32_t* __restrict__ cnt_out,
                                                            int64_t* __restrict__ first_out, int32_t* __restrict__ len_out,
                                                            int32_t* status) {
  constexpr int RW = 2;                                                   // roots of a warp
  const int lane = threadIdx.x & 31;
  const int64_t root0 = ((blockIdx.x * (int64_t)blockDim.x + threadIdx.x) >> 5) * RW;
  if (root0 >= n) return;
  int64_t base[RW];
  uint32_t lo[RW], hi[RW];                                                // the bound lies in [lo, hi] behind base
  double t[RW];
  int node[RW];
#pragma unroll
  for (int i = 0; i < RW; ++i) {
    node[i] = root0 + i < n ? nodes[root0 + i] : -1;
    t[i] = root0 + i < n ? times[root0 + i] : 0.0;
  }
#pragma unroll
  for (int i = 0; i < RW; ++i) {
    const bool known = node[i] >= 0 && node[i] < N;
    base[i] = known ? indptr[node[i]] : 0;
    int64_t end = known ? indptr[node[i] + 1] : -1;
    // a node outside the graph, or a slice outside the entries: reported, nothing visible
    if (base[i] < 0 || end < base[i] || end > P || end - base[i] > 0x7fffffff) {
      if (lane == 0 && root0 + i < n) atomicMax(status, 4);
      base[i] = end = 0;
    }
    lo[i] = 0;
    hi[i] = (uint32_t)(end - base[i]);
  }
  while (hi[0] - lo[0] > 32 || hi[1] - lo[1] > 32) {
    uint32_t idx[RW];
    bool below[RW];
#pragma unroll
    for (int i = 0; i < RW; ++i) {
      idx[i] = lo[i] + (uint32_t)(lane + 1) * ((hi[i] - lo[i]) / 33);     // in [lo, hi) and ascending for ranges of 33 and more
      below[i] = hi[i] - lo[i] > 32 && (g_ts + base[i])[idx[i]] < t[i];
    }
#pragma unroll
    for (int i = 0; i < RW; ++i) {
      if (hi[i] - lo[i] <= 32) continue;
      const int c = __popc(__ballot_sync(FULL, below[i]));
      const uint32_t idx_hi = __shfl_sync(FULL, idx[i], c < 32 ? c : 31); // first probe with ts >= t
      const uint32_t idx_lo = __shfl_sync(FULL, idx[i], c > 0 ? c - 1 : 0);   // last probe with ts < t
      if (c < 32) hi[i] = idx_hi;
      if (c > 0) lo[i] = idx_lo + 1;
    }
  }
  bool below[RW];
#pragma unroll
  for (int i = 0; i < RW; ++i) below[i] = (uint32_t)lane < hi[i] - lo[i] && (g_ts + base[i])[lo[i] + lane] < t[i];
  int len[RW], nw[RW], ns[RW];
  const int slots = window + sinks;
#pragma unroll
  for (int i = 0; i < RW; ++i) {
    len[i] = (int)lo[i] + __popc(__ballot_sync(FULL, below[i]));
    nw[i] = min(len[i], window);
    ns[i] = min(len[i] - nw[i], sinks);
    if (lane == 0 && root0 + i < n) {
      if (first_out) first_out[root0 + i] = base[i];
      if (len_out) len_out[root0 + i] = len[i];
      if (cnt_out) cnt_out[root0 + i] = nw[i] + ns[i];
    }
  }
  if (!nbr_out && !eid_out && !ts_out) return;
  for (int j = lane; j < slots; j += 32) {
    int nb[RW], ev[RW];
    double tt[RW];
#pragma unroll
    for (int i = 0; i < RW; ++i) {
      const bool in = j < nw[i] + ns[i];
      const int64_t e = j < nw[i] ? base[i] + len[i] - 1 - j : base[i] + (j - nw[i]);
      nb[i] = nbr_out && in ? __ldg(g_nbr + e) : -1;
      ev[i] = eid_out && in ? __ldg(g_eid + e) : -1;
      tt[i] = ts_out && in ? __ldg(g_ts + e) : 0.0;
    }
#pragma unroll
    for (int i = 0; i < RW; ++i) {
      if (root0 + i >= n) continue;
      const int64_t at = (root0 + i) * slots + j;
      if (nbr_out) nbr_out[at] = nb[i];
      if (eid_out) eid_out[at] = ev[i];
      if (ts_out) ts_out[at] = tt[i];
    }
  }
}

}  // namespace

extern "C" int tgnn_sample_window(const int64_t* indptr, const int32_t* nbr, const int32_t* eid, const double* ts, int64_t num_nodes,
                                  int64_t num_entries, const int32_t* nodes, const double* times, int64_t n, int window, int sinks,
                                  int32_t* nbr_out, int32_t* eid_out, double* ts_out, int32_t* cnt_out, int64_t* first_out,
                                  int32_t* len_out, int32_t* status, void* stream, char* err_host, int64_t err_size) {
  const char* who = "tgnn_sample_window";
  if (n < 0 || num_nodes < 0 || num_entries < 0 || window < 0 || sinks < 0 || (int64_t)window + sinks < 1)
    return fail(err_host, err_size, TGNN_EINVAL, "%s: size out of range (window and sinks hold one slot at least)", who);
  if (n > 0x7fffffff) return fail(err_host, err_size, TGNN_ECAPACITY, "%s: n beyond int32", who);
  if ((nbr_out || eid_out || ts_out) && (int64_t)window + sinks > 65536)
    return fail(err_host, err_size, TGNN_ECAPACITY, "%s: more than 65536 slots", who);
  if (!status || (n > 0 && (!nodes || !times || (num_nodes > 0 && !indptr) || (num_entries > 0 && !ts))))
    return fail(err_host, err_size, TGNN_EINVAL, "%s: null pointer", who);
  if (num_entries > 0 && ((nbr_out && !nbr) || (eid_out && !eid)))
    return fail(err_host, err_size, TGNN_EINVAL, "%s: slots of an array that is not given", who);
  if ((((uintptr_t)indptr | (uintptr_t)ts | (uintptr_t)times | (uintptr_t)ts_out | (uintptr_t)first_out) & 7) ||
      (((uintptr_t)nbr | (uintptr_t)eid | (uintptr_t)nodes | (uintptr_t)nbr_out | (uintptr_t)eid_out | (uintptr_t)cnt_out |
        (uintptr_t)len_out | (uintptr_t)status) & 3))
    return fail(err_host, err_size, TGNN_EINVAL, "%s: a pointer is not aligned to its element", who);
  if (n == 0) return TGNN_OK;
  const unsigned grid = (unsigned)((n + 7) / 8);                           // 4 warps of two roots
  sample_window_kernel<<<grid, 128, 0, (cudaStream_t)stream>>>(indptr, nbr, eid, ts, num_nodes, num_entries, nodes, times, (int)n, window,
                                                              sinks, nbr_out, eid_out, ts_out, cnt_out, first_out, len_out, status);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return fail(err_host, err_size, TGNN_ECUDA, "%s: %s", who, cudaGetErrorString(e));
  return TGNN_OK;
}
