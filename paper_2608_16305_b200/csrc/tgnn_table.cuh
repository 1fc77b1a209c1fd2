// What the node-table operators share (lookup, destination loss, AdamW): groups of values of a row as words, launches in a chain.
#pragma once
#include "tgnn_history.cuh"

namespace tgnn_table {

using tgnn_history::elem_bytes;
using tgnn_history::fail;
using tgnn_history::FULL;
using tgnn_history::known_dtype;
using tgnn_history::num_sms;

// Pairs of 16-bit values.
template <typename T>
struct Pair { typedef T type; };
template <>
struct Pair<__nv_bfloat16> { typedef __nv_bfloat162 type; };
template <>
struct Pair<__half> { typedef __half2 type; };
__device__ __forceinline__ float2 widen(__nv_bfloat162 x) { return __bfloat1622float2(x); }
__device__ __forceinline__ float2 widen(__half2 x) { return __half22float2(x); }
__device__ __forceinline__ void narrow(float a, float b, __nv_bfloat162* to) { *to = __floats2bfloat162_rn(a, b); }
__device__ __forceinline__ void narrow(float a, float b, __half2* to) { *to = __floats2half2_rn(a, b); }

// V values of type T as one access (V * sizeof(T) up to 16 bytes, the address a multiple of that).
template <typename T, int V>
struct Group {
  typename tgnn_history::Vec<V * (int)sizeof(T)>::type w;
  __device__ __forceinline__ void get(float* x) const {
    const T* t = reinterpret_cast<const T*>(&w);
    if constexpr (sizeof(T) == 2 && V > 1) {                                    // two at a time
#pragma unroll
      for (int i = 0; i < V; i += 2) {
        const float2 f = widen(reinterpret_cast<const typename Pair<T>::type*>(t + i)[0]);
        x[i] = f.x;
        x[i + 1] = f.y;
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = tgnn_history::to_float<T>(t[i]);
    }
  }
  __device__ __forceinline__ void set(const float* x) {
    T* t = reinterpret_cast<T*>(&w);
    if constexpr (sizeof(T) == 2 && V > 1) {
#pragma unroll
      for (int i = 0; i < V; i += 2) narrow(x[i], x[i + 1], reinterpret_cast<typename Pair<T>::type*>(t + i));
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) t[i] = tgnn_history::from_float<T>(x[i]);
    }
  }
};

// Kernels of one call are launched as a chain: a kernel may be put on the device while the one before it ends, and chain_wait holds it until
// that one's results are visible.  Every kernel of a chain waits before it touches global memory, so the order reaches back to the first.
__device__ __forceinline__ void chain_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void chain_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

struct Chain {
  cudaStream_t stream;
  cudaError_t e = cudaSuccess;
  bool first = true;
  explicit Chain(void* s) : stream((cudaStream_t)s) {}
  template <typename... P, typename... A>
  void operator()(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, A... args) {
    if (e != cudaSuccess) return;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = first ? 0 : 1;
    e = cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
    first = false;
  }
  int end(const char* who, char* err, int64_t size) {
    if (e == cudaSuccess) return TGNN_OK;
    cudaGetLastError();
    return fail(err, size, TGNN_ECUDA, "%s: %s", who, cudaGetErrorString(e));
  }
};

__host__ __device__ inline int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

}  // namespace tgnn_table
