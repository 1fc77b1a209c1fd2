// Slot attention: entry points and the forward pass's kernels.  slot_attend.cuh has the mathematics; the backward pass's kernels of each type
// are compiled in a file of their own, which is a minute instead of three.
#include "slot_attend.cuh"

using namespace tgnn_slots;

extern "C" {

int tgnn_slot_attend(const void* q, const void* k, const void* v, int dtype, int64_t n, int slots, int heads, int kv_heads, int dim,
                     const int32_t* cnt, const float* bias, int num_buckets, const double* bounds, const double* times, const double* ts,
                     float scale, void* out, void* stream, char* err_host, int64_t err_size) {
  SlotArgs a = args_of(q, k, v, n, slots, heads, kv_heads, dim, cnt, bias, num_buckets, bounds, times, ts, scale);
  a.out = out;
  return run<false>("tgnn_slot_attend", a, dtype, out, nullptr, nullptr, stream, err_host, err_size);
}

int64_t tgnn_slot_attend_scratch(int64_t n, int heads, int num_buckets) {
  if (n < 0 || heads < 1 || heads > 256 || num_buckets < 0 || num_buckets > kMaxBuckets) return -1;
  return 2 * (n < MAX_BLOCKS ? n : (int64_t)MAX_BLOCKS) * heads * num_buckets;
}

int tgnn_slot_attend_backward(const void* q, const void* k, const void* v, int dtype, int64_t n, int slots, int heads, int kv_heads, int dim,
                              const int32_t* cnt, const float* bias, int num_buckets, const double* bounds, const double* times,
                              const double* ts, float scale, const void* dout, void* dq, void* dk, void* dv, float* dbias, float* scratch,
                              void* stream, char* err_host, int64_t err_size) {
  SlotArgs a = args_of(q, k, v, n, slots, heads, kv_heads, dim, cnt, bias, num_buckets, bounds, times, ts, scale);
  a.dout = dout;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  return run<true>("tgnn_slot_attend_backward", a, dtype, dq, dbias, scratch, stream, err_host, err_size);
}

}  // extern "C"
